// Causal attention over packed prompts.
//
// A workgroup takes 128 query rows, a wave 32 of them, and walks the keys 64 at a time.  Keys and values go to LDS
// by LDS-DMA (no registers), the next tile's while this one is worked on.  Products are v_mfma_f32_32x32x16_f16:
//   scores  S^T = K Q^T: A = keys from LDS, B = queries, which stay in registers.  Lane (column q, half h) receives the scores of its query
//           with keys 8 i + 4 h .. + 3, which packed to fp16 are the B operand of the second product as they stand
//   output  O^T = V^T P^T: A = values by the transposing LDS read, in the same order of keys
// so weights never leave the lane.  A row of LDS is a token's head; its 16-byte pieces are permuted by the token's number, so that both kinds of
// reads (16 tokens at one piece, 4 tokens at 4 pieces) touch all banks evenly.
// Softmax: powers of 2 relative to a row's reference, which moves only when a score is more than 2^8 beyond it (fp16 holds the weights all the same), so most tiles need
// no exchange between lanes and no scaling of the sums.
// Bound: the matrix pipes and, beside them, the softmax's vector instructions; two workgroups on a CU, so that one's products run beside the other's softmax.
// Rounding: scores, statistics and sums in 32 bits; weights become fp16 for the second product, whose matrix instructions take no more (2^-11 of each, or 2^-32 of the reference where that is
// more: at the reference a weight is 2^7, so that fp16 has its range where weights are), and their sum is of the rounded ones, so that weights add up to 1.
// Measured: 16384 tokens, 32 heads of 128 on 8 key heads 2.01 to 2.16 ms from card to card, 1.02 to 1.09 PFLOP/s: the matrix pipes are busy 61 % of the time and the chip's power sets the clock (1.75 GHz; the same
// on zeros 1.48 ms).  2048 tokens with 32 heads of 128 47 to 52 us; 11 packed prompts of up to 1500 with 32 heads of 64 on 8 55 to 57 us.
#include "tl_attn.hpp"

#include <type_traits>

namespace tl {
namespace {

constexpr float kInf = __builtin_inff();
constexpr int kTile = 64;                 // keys

// LDS addresses are 32-bit numbers here
#pragma clang diagnostic ignored "-Wint-to-pointer-cast"

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef __attribute__((address_space(3))) f16x8 lds_f16x8;

__device__ inline float finite(float x) { return x == -kInf ? 0.0f : x; }
__device__ inline float power(float x) { return __builtin_amdgcn_exp2f(x); }
// What a row's sums are multiplied by.  Every row sees a key, so its weights add up to 2^kLift at least, unless all its scores are -infinity, whose softmax is 0 / 0.
__device__ inline float share(float l) { return l > 0.0f ? 1.0f / l : __builtin_nanf(""); }

__device__ inline uint32_t lds_address(const void* p)
{
    return uint32_t(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)p));
}

// 16 bytes a lane from base + off to LDS, the lanes' side by side.
__device__ inline void transfer(const void* base, uint32_t off, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory", "m0");
}

// Where piece c (16 bytes) of token r stands in its row.
template <int DP>
__device__ inline int piece(int r, int c)
{
    if constexpr (DP == 128) return c ^ (((r & 3) << 2) | ((r >> 2) & 3));
    else return c ^ ((((r >> 1) & 1) << 2) | ((r >> 2) & 3));
}

// Blocks of `rows` query rows of all sequences (64 at most), those with most keys before others: the one in that place.  What is heavy begins early, so that the chip is
// full until the end; with `two` to a compute unit, where all fit at once, the second half comes in the opposite order, so that a heavy one shares its unit with a light one.
__device__ inline Item nth_longest(const PromptArgs& a, int rows, int heads, bool two, int place)
{
    const int lane = threadIdx.x & 63;
    const int n = lane < a.b.seqs ? span(a.b, lane).n : 0, blocks = (n + rows - 1) / rows;
    auto from = [&](int j) {                                 // blocks with numbers from j on
        return wave_sum(blocks > j ? blocks - j : 0);
    };
    const int all = from(0);
    if (place >= all) return {-1, 0};
    const int half = 256 / heads;
    if (two && int64_t(all) * heads <= 512 && place >= half) place = all - 1 - (place - half);
    if (a.b.seqs == 1) return {0, all - 1 - place};
    // the largest number j with more than `place` blocks from j on
    int lo = 0, hi = 1;
    while (from(hi) > place) { lo = hi; hi *= 2; }
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (from(mid) > place) lo = mid;
        else hi = mid;
    }
    int skip = place - from(lo + 1);
    uint64_t there = __ballot(blocks > lo);
    while (skip-- > 0) there &= there - 1;
    return {int(__builtin_ctzll(there)), lo};
}

// What a workgroup takes: a block of `rows` query rows of a sequence, and one of `heads` heads or groups of heads.
struct Where { int seq, block, head; };
__device__ inline Where where(const PromptArgs& a, int rows, int heads, bool two)
{
    // heads that share keys go to one chiplet (workgroups are dealt to the 8 of them in turn); the rows with most keys first
    int h = int(blockIdx.x) % heads;
    const int place = int(blockIdx.x) / heads, places = int(gridDim.x) / heads;
    Item it{places - 1 - place, 0};
    if (a.b.start && a.b.seqs <= 64) it = nth_longest(a, rows, heads, two, place);
    else if (a.b.start) it = find_item(a.b, places - 1 - place, rows, 1);
    if (heads % 8 == 0) h = (h & 7) * (heads >> 3) + (h >> 3);
    return {__builtin_amdgcn_readfirstlane(it.seq), __builtin_amdgcn_readfirstlane(it.i), h};
}

// A row's queries, turned round where the scale is negative, or 0: so that the largest product is the largest score.
template <int KK>
__device__ inline void load_queries(const PromptArgs& a, const _Float16* from, int half, f16x8 (&q)[KK])
{
#pragma unroll
    for (int k = 0; k < KK; ++k) {
        const int c = 2 * k + half;
        q[k] = *reinterpret_cast<const f16x8*>(from + (c < (a.dim >> 3) ? c : 0) * 8);
        if (c >= (a.dim >> 3)) q[k] = f16x8{0, 0, 0, 0, 0, 0, 0, 0};
    }
    if (a.scale == 0.0f) {
#pragma unroll
        for (int k = 0; k < KK; ++k) q[k] *= _Float16(0.0f);              // an infinity or a NaN stays one
    }
    if (a.scale < 0.0f) {
#pragma unroll
        for (int k = 0; k < KK; ++k) q[k] = -q[k];
    }
}

// Two fp16: ones in the place of each that is an infinity or a NaN (whose exponent of ones carries into the sign's place).
__device__ inline uint32_t only_finite(uint32_t two) { return ((((two & 0x7c007c00u) + 0x04000400u) & 0x80008000u) >> 15) * 0xffffu; }

// 128 query rows a workgroup: of one head, or 64 or 32 of each of two or four HEADS that share their keys, which leaves fewer rows behind a sequence's end and less of the last tiles masked.
template <int DP, int HEADS>
__global__ __launch_bounds__(256, 2) void prompt_kernel(PromptArgs a)
{
    constexpr int NW = 4;                                    // waves, 32 rows each
    constexpr int kRow = DP * 2, kPieces = DP / 8, kBytes = kTile * kRow;
    constexpr int kSteps = kBytes / (NW * 1024);             // transfers of a wave for keys, and as many for values
    constexpr int kRows1 = 1024 / kRow;                      // tokens of a transfer
    constexpr int KK = DP / 16, DT = DP / 32;
    constexpr int kRows = 32 * NW / HEADS;                   // of a head
    __shared__ __attribute__((aligned(1024))) unsigned char lds[2][2][kBytes];
    __shared__ int strange[2][NW];                           // whether the values that a wave brought hold an infinity or a NaN
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5;

    const Where where_ = where(a, kRows, a.q_heads / HEADS, true);
    const int seq = where_.seq, h = where_.head * HEADS + wave % HEADS;
    if (seq < 0) return;
    const Span sp = span(a.b, seq);
    const int n = __builtin_amdgcn_readfirstlane(sp.n), first = __builtin_amdgcn_readfirstlane(sp.first);
    const int q0 = where_.block * kRows;
    if (q0 >= n) return;
    const int g = h / a.group;
    const int row0 = q0 + wave / HEADS * 32, row = row0 + l32;       // this lane's query in the sequence
    const int pieces = a.dim >> 3;
    const float scale = a.scale == 0.0f ? 1.0f : fabsf(a.scale);      // with queries that are turned round, or 0: the largest product is the largest score

    if (pieces < kPieces) {                                  // dimensions beyond the head are never transferred
        for (int i = threadIdx.x; i < 4 * kBytes / 16; i += 64 * NW) reinterpret_cast<u32x4*>(&lds[0][0][0])[i] = u32x4{0, 0, 0, 0};
        __syncthreads();
    }
    const int most = q0 + kRows < n ? q0 + kRows : n;        // keys that the workgroup sees
    const int tiles = (most + kTile - 1) / kTile, full = q0 / kTile & ~1;     // the first ones without a mask, both buffers as often
    const char* const kbase = reinterpret_cast<const char*>(a.k.p + int64_t(first) * a.k.token + int64_t(g) * a.k.head);
    const char* const vbase = reinterpret_cast<const char*>(a.v.p + int64_t(first) * a.v.token + int64_t(g) * a.v.head);
    const uint32_t kstride = uint32_t(a.k.token) * 2u, vstride = uint32_t(a.v.token) * 2u;
    const uint32_t lds0 = lds_address(&lds[0][0][0]) + wave * kSteps * 1024;
    uint32_t koff[kSteps], voff[kSteps];                     // this lane's pieces of a whole tile
    bool mine[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int r = (wave * kSteps + i) * kRows1 + lane / kPieces, c = piece<DP>(r, lane % kPieces);
        koff[i] = uint32_t(r) * kstride + c * 16;
        voff[i] = uint32_t(r) * vstride + c * 16;
        mine[i] = c < pieces;
    }
    auto fetch = [&](int t, int buf) {
        if (t > tiles - 1) t = tiles - 1;                    // so that the number of transfers on their way is always the same
        const char* const kb = kbase + int64_t(t) * kTile * kstride;
        const char* const vb = vbase + int64_t(t) * kTile * vstride;
        const int last = n - 1 - t * kTile;
        if (last >= kTile - 1) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
                if (mine[i]) {
                    transfer(kb, koff[i], lds0 + buf * 2 * kBytes + i * 1024);
                    transfer(vb, voff[i], lds0 + (buf * 2 + 1) * kBytes + i * 1024);
                }
        } else {
            // tokens behind the sequence are masked: the last one again, no NaN that is not there
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int r = (wave * kSteps + i) * kRows1 + lane / kPieces;
                const uint32_t back = uint32_t(r > last ? r - last : 0);
                if (mine[i]) {
                    transfer(kb, koff[i] - back * kstride, lds0 + buf * 2 * kBytes + i * 1024);
                    transfer(vb, voff[i] - back * vstride, lds0 + (buf * 2 + 1) * kBytes + i * 1024);
                }
            }
        }
    };

    fetch(0, 0);
    f16x8 q[KK];
    load_queries<KK>(a, a.q.p + int64_t(first + (row < n ? row : n - 1)) * a.q.token + int64_t(h) * a.q.head, half, q);
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    bool left_out = false;                                   // infinities and NaN of values, of which some row must not hear
    float m = -kInf, l = 0.0f;

    // Where this lane's pieces stand in a tile: keys 2 k + half of token l32, values of 32 dimensions d and tokens 8 e + 4 half + 0 .. 3.  The rest of an
    // address is a multiple of a row count that the permutation does not see, and goes into the instruction.
    const uint32_t base = lds_address(&lds[0][0][0]);
    uint32_t ka[KK], va[DT][2];
#pragma unroll
    for (int k = 0; k < KK; ++k) ka[k] = base + l32 * kRow + piece<DP>(l32, 2 * k + half) * 16;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = e * 8 + half * 4 + ((lane & 15) >> 2), c = d * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
            va[d][e] = base + kBytes + r * kRow + piece<DP>(r, c) * 16 + (lane & 1) * 8;
        }

    // One tile, `at` bytes behind the first; MASKED: some row of the wave does not see all of it.
    auto work = [&](int t, auto at, auto some) {
        constexpr bool MASKED = decltype(some)::value;
        constexpr int B = decltype(at)::value / (2 * kBytes);
        f32x16 s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < KK; ++k)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const lds_f16x8*)(ka[k] + (at + b * 32 * kRow)), q[k], s[b], 0, 0, 0);
        // reads six products ahead: one at a time, each product would wait for its read
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int i = 0; i < 2 * KK; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        const int seen = row - t * kTile - 4 * half;         // key 32 b + 8 (i / 4) + 4 half + i % 4 is seen up to the row's own number
        if constexpr (MASKED) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * b + 8 * (i >> 2) + (i & 3) > seen) s[b][i] = -kInf;
        }
        float mx = -kInf;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, s[b][i]), s[b][i + 1]);
        mx = mx == -kInf ? mx : __builtin_fmaf(mx, scale, -kLift);
        if (__any(mx > m + kSlack)) {
            // each row by itself: what one row sees does not change how another is rounded
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float to = mx > m + kSlack ? mx : m;
            const float f = power(m - finite(to));
            l *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= f;
            m = to;
        }
        const float mb = finite(m);
        f16x8 w[4];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                w[b * 2 + (i >> 3)][i & 7] = _Float16(power(__builtin_fmaf(s[b][i], scale, -mb)));
            }
        // the sum of the weights as they are rounded, two at a time
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 8; i += 2) l = __builtin_amdgcn_fdot2(f16x2{w[u][i], w[u][i + 1]}, f16x2{_Float16(1.0f), _Float16(1.0f)}, l, false);
        // values of 16 keys and 32 dimensions, in the order of the weights
        auto values = [&](int u, int d) {
            union { f16x8 v; i16x4 h[2]; } x;
#pragma unroll
            for (int e = 0; e < 2; ++e) x.h[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(va[d][e] + (at + u * 16 * kRow)));
            return x.v;
        };
        if constexpr (MASKED) {
            // A weight of 0 does not take an infinity or a NaN out of a sum: where the tile has any, they are left out here and added at the end.
            bool odd = false;
#pragma unroll
            for (int v = 0; v < NW; ++v) odd |= strange[B][v] != 0;
            if (__any(odd)) {
                left_out = true;
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        union { f16x8 v; uint32_t w[4]; } x{values(u, d)};
#pragma unroll
                        for (int i = 0; i < 4; ++i) x.w[i] &= ~only_finite(x.w[i]);
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x.v, w[u], o[d], 0, 0, 0);
                    }
                return;
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(values(u, d), w[u], o[d], 0, 0, 0);
    };

    // the next tile is there, and all waves are done with the last one
    auto arrived = [&] {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    // looks at the values that this wave has transferred to a buffer, before others may read them
    auto look = [&](int buf) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        f16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
            zero += *(const lds_f16x8*)(base + kBytes + (wave * kSteps + i) * 1024 + lane * 16 + buf * 2 * kBytes) * _Float16(0.0f);
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) odd |= !(zero[i] == _Float16(0.0f));
        odd = __any(odd);
        if (lane == 0) strange[buf][wave] = odd;
    };
    if (full == 0) look(0);
    arrived();
    // Tiles that all rows of the workgroup see, two at a time; while a tile is worked on, the next is on its way.
    int t = 0;
    auto whole = [&](auto buf) {
        constexpr int B = decltype(buf)::value;
        fetch(t + 1, B ^ 1);
        work(t, std::integral_constant<int, B * 2 * kBytes>{}, std::false_type{});
        ++t;
        if (B == 1 && t == full) look(0);
        arrived();
    };
    // tiles that some row does not see, or not all of
    auto last = [&](auto buf) {
        constexpr int B = decltype(buf)::value;
        if (t >= tiles) return;
        fetch(t + 1, B ^ 1);
        if (t * kTile <= row0 + 31) work(t, std::integral_constant<int, B * 2 * kBytes>{}, std::true_type{});      // behind, no row of this wave sees a key
        ++t;
        if (t < tiles) look(B ^ 1);
        arrived();
    };
    constexpr std::integral_constant<int, 0> kFirst{};
    constexpr std::integral_constant<int, 1> kSecond{};
    while (t < full) {
        whole(kFirst);
        whole(kSecond);
    }
    last(kFirst);
    last(kSecond);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();

    if (left_out) {
        // values of the tokens that only some rows see, once more: an infinity or a NaN goes to the rows that see it
        for (int key = full * kTile; key < most; ++key) {
            const _Float16* v = reinterpret_cast<const _Float16*>(vbase) + int64_t(key) * a.v.token;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = d * 32 + i * 8 + half * 4;
                    const f16x4 x = *reinterpret_cast<const f16x4*>(v + (at < a.dim ? at : 0));
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (key <= row && !(__builtin_fabsf16(x[j]) < _Float16(kInf))) o[d][i * 4 + j] += float(x[j]);
                }
        }
    }
    l += __shfl_xor(l, 32);
    const float f = share(l);
    // Through LDS, which nobody reads any more, so that whole rows are written at once.  A row has 16 bytes beside it: rows begin in different banks.
    constexpr int kOut = kRow + 16;
    static_assert(NW * 32 * kOut <= 4 * kBytes, "a workgroup's rows in LDS");
    unsigned char* const rows = &lds[0][0][0] + wave * 32 * kOut;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f16x4 y;
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = _Float16(o[d][i * 4 + j] * f);
            *reinterpret_cast<f16x4*>(rows + l32 * kOut + (d * 32 + i * 8 + half * 4) * 2) = y;
        }
    // a wave reads what it wrote itself
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    const int c = lane % kPieces;
#pragma unroll
    for (int i = 0; i < 32 / kRows1; ++i) {
        const int r = i * kRows1 + lane / kPieces;
        if (row0 + r < n && c < pieces)
            *reinterpret_cast<f16x8*>(a.out.p + int64_t(first + row0 + r) * a.out.token + int64_t(h) * a.out.head + c * 8) = *reinterpret_cast<const f16x8*>(rows + r * kOut + c * 16);
    }
}

// The same for 64 query rows a workgroup, 32 a wave, S waves for each of them, which deal tiles of 32 keys among themselves and join their sums in LDS at the end: for few rows
// with many keys (S = 4), where workgroups of 128 rows with all their keys leave most of the chip idle, and for many sequences of a few tokens (S = 1), where they are idle themselves.
// Bound: with heads of 64 a round (64 rows, 128 keys) takes 0.77 us, 0.58 of it without the transfers and 0.60 without the products: the one barrier a round lets them overlap little,
// and more rounds in LDS ahead did not help.  Measured: one head of 64, 14587 tokens 92 us; 8 of 128, 2048 tokens 29 us.
template <int DP, int S>
__global__ __launch_bounds__(128 * S, DP == 64 ? 4 : 2) void narrow_kernel(PromptArgs a)
{
    constexpr int R = 2, kKeys = 32 * S, kRow = DP * 2, kPieces = DP / 8, kBytes = kKeys * kRow, kSteps = kBytes / (R * S * 1024), kRows1 = 1024 / kRow;
    constexpr int KK = DP / 16, DT = DP / 32;
    constexpr int kSum = DP + 4;                             // a row's sums in LDS, so that rows begin in different banks
    constexpr int kLds = R * S * 32 * kSum * 4 > 4 * kBytes ? R * S * 32 * kSum * 4 : 4 * kBytes;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kLds];
    __shared__ float stats[S][32 * R][2];
    __shared__ int strange[R];                               // whether values that only some of the rows see hold an infinity or a NaN
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5, rw = wave % R, kw = wave / R;
    const Where at = where(a, 32 * R, a.q_heads, DP == 64);
    if (at.seq < 0) return;
    const Span sp = span(a.b, at.seq);
    const int n = __builtin_amdgcn_readfirstlane(sp.n), first = __builtin_amdgcn_readfirstlane(sp.first), h = at.head, g = h / a.group;
    const int q0 = at.block * (32 * R), own = at.block * R + rw, row = own * 32 + l32, pieces = a.dim >> 3;
    if (q0 >= n) return;
    const int whole = (n + 31) / 32, tiles = (at.block + 1) * R < whole ? (at.block + 1) * R : whole, rounds = (tiles + S - 1) / S;
    const float scale = a.scale == 0.0f ? 1.0f : fabsf(a.scale);
    if (pieces < kPieces) {                                  // dimensions beyond the head are never transferred
        for (int i = threadIdx.x; i < 4 * kBytes / 16; i += 64 * R * S) reinterpret_cast<u32x4*>(lds)[i] = u32x4{0, 0, 0, 0};
        __syncthreads();
    }
    const char* const kbase = reinterpret_cast<const char*>(a.k.p + int64_t(first) * a.k.token + int64_t(g) * a.k.head);
    const char* const vbase = reinterpret_cast<const char*>(a.v.p + int64_t(first) * a.v.token + int64_t(g) * a.v.head);
    const uint32_t kstride = uint32_t(a.k.token) * 2u, vstride = uint32_t(a.v.token) * 2u;
    const uint32_t base = lds_address(lds);
    auto fetch = [&](int round, int buf) {
        const char* const kb = kbase + int64_t(round) * kKeys * kstride;
        const char* const vb = vbase + int64_t(round) * kKeys * vstride;
        const int last = n - 1 - round * kKeys;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            int r = (wave * kSteps + i) * kRows1 + lane / kPieces;
            const int c = piece<DP>(r, lane % kPieces);
            if (r > last) r = last;                          // tokens behind the sequence are masked: the last one again, no NaN that is not there
            if (c < pieces) {
                transfer(kb, uint32_t(r) * kstride + c * 16, base + buf * 2 * kBytes + (wave * kSteps + i) * 1024);
                transfer(vb, uint32_t(r) * vstride + c * 16, base + (buf * 2 + 1) * kBytes + (wave * kSteps + i) * 1024);
            }
        }
    };
    fetch(0, 0);
    f16x8 q[KK];
    load_queries<KK>(a, a.q.p + int64_t(first + (row < n ? row : n - 1)) * a.q.token + int64_t(h) * a.q.head, half, q);
    const uint32_t mine = base + kw * 32 * kRow;
    uint32_t ka[KK], va[DT][2];
#pragma unroll
    for (int k = 0; k < KK; ++k) ka[k] = mine + l32 * kRow + piece<DP>(l32, 2 * k + half) * 16;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = e * 8 + half * 4 + ((lane & 15) >> 2), c = d * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
            va[d][e] = mine + kBytes + r * kRow + piece<DP>(r, c) * 16 + (lane & 1) * 8;
        }
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    float m = -kInf, l = 0.0f;
    bool left_out = false;
    auto work = [&](int t, auto buf) {
        constexpr int AT = decltype(buf)::value * 2 * kBytes;
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < KK; ++k) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const lds_f16x8*)(ka[k] + AT), q[k], s, 0, 0, 0);
        // all reads before the products: 97 us for the one head, 92
        __builtin_amdgcn_sched_group_barrier(0x100, KK, 0);
        __builtin_amdgcn_sched_group_barrier(0x8, KK, 0);
        bool odd = false;
        if (t == own) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i >> 2) + 4 * half + (i & 3) > l32) s[i] = -kInf;
            f16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 32 * kRow / 1024; ++i) zero += *(const lds_f16x8*)(mine + kBytes + AT + i * 1024 + lane * 16) * _Float16(0.0f);
#pragma unroll
            for (int i = 0; i < 8; ++i) odd |= !(zero[i] == _Float16(0.0f));
            odd = __any(odd);
            left_out = odd;
        }
        float mx = -kInf;
#pragma unroll
        for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, s[i]), s[i + 1]);
        mx = mx == -kInf ? mx : __builtin_fmaf(mx, scale, -kLift);
        if (__any(mx > m + kSlack)) {
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float to = mx > m + kSlack ? mx : m;
            const float f = power(m - finite(to));
            l *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= f;
            m = to;
        }
        const float mb = finite(m);
        f16x8 w[2];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i >> 3][i & 7] = _Float16(power(__builtin_fmaf(s[i], scale, -mb)));
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 8; i += 2) l = __builtin_amdgcn_fdot2(f16x2{w[u][i], w[u][i + 1]}, f16x2{_Float16(1.0f), _Float16(1.0f)}, l, false);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                union { f16x8 v; i16x4 h[2]; uint32_t w[4]; } x;
#pragma unroll
                for (int e = 0; e < 2; ++e) x.h[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(va[d][e] + (AT + u * 16 * kRow)));
                if (odd) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x.w[i] &= ~only_finite(x.w[i]);
                }
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x.v, w[u], o[d], 0, 0, 0);
            }
    };
    auto turn = [&](int round, auto buf) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __syncthreads();                                     // these keys are there, and nobody reads from the other buffer any more
        if (round + 1 < rounds) fetch(round + 1, decltype(buf)::value ^ 1);
        const int t = round * S + kw;
        if (t <= own) work(t, buf);
    };
    for (int round = 0; round < rounds; round += 2) {
        turn(round, std::integral_constant<int, 0>{});
        if (round + 1 < rounds) turn(round + 1, std::integral_constant<int, 1>{});
    }
    l += __shfl_xor(l, 32);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __syncthreads();
    // The waves' sums meet in LDS, where keys and values were.
    float* const sums = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4*>(sums + ((kw * R + rw) * 32 + l32) * kSum + d * 32 + i * 8 + half * 4) =
                f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    if (half == 0) {
        stats[kw][rw * 32 + l32][0] = m;
        stats[kw][rw * 32 + l32][1] = l;
    }
    if (own % S == kw && lane == 0) strange[rw] = left_out;  // the wave of the keys that are masked for some
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * R * kPieces; i += 64 * R * S) {
        const int r = i / kPieces, c = i % kPieces;
        if (q0 + r >= n || c >= pieces) continue;
        float M = -kInf, L = 0.0f;
#pragma unroll
        for (int v = 0; v < S; ++v) M = fmaxf(M, stats[v][r][0]);
        M = finite(M);
        f32x4 x[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int v = 0; v < S; ++v) {
            const float f = power(stats[v][r][0] - M);
            const float* from = sums + (v * R * 32 + r) * kSum + c * 8;
            L += stats[v][r][1] * f;
            x[0] += *reinterpret_cast<const f32x4*>(from) * f;
            x[1] += *reinterpret_cast<const f32x4*>(from + 4) * f;
        }
        const float f = share(L);
        f16x8 y;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float sum = x[j >> 2][j & 3];
            if (strange[r >> 5]) {
                // values of the tokens that only some rows see, once more: an infinity or a NaN goes to the rows that see it
                for (int key = q0 + (r & ~31); key <= q0 + r; ++key) {
                    const float v = float(reinterpret_cast<const _Float16*>(vbase)[int64_t(key) * a.v.token + c * 8 + j]);
                    if (!(fabsf(v) < kInf)) sum += v;
                }
            }
            y[j] = _Float16(sum * f);
        }
        *reinterpret_cast<f16x8*>(a.out.p + int64_t(first + q0 + r) * a.out.token + int64_t(h) * a.out.head + c * 8) = y;
    }
}

}  // namespace

hipError_t launch_prompt(const PromptArgs& a, hipStream_t s)
{
    const auto grid = [&](int rows) { return (a.b.start ? a.b.tokens / rows + a.b.seqs : a.b.seqs) * a.q_heads; };
    const unsigned small = unsigned(grid(64));
    // about as many of 64 rows have work
    const int64_t busy = a.b.start ? (a.b.tokens + 32 * int64_t(a.b.seqs)) / 64 * a.q_heads : small;
    const auto heads_together = [&](auto n) {
        constexpr int N = decltype(n)::value;
        const unsigned groups = unsigned(grid(128 / N) / N);
        if (a.dim <= 64) prompt_kernel<64, N><<<groups, 256, 0, s>>>(a);
        else prompt_kernel<128, N><<<groups, 256, 0, s>>>(a);
    };
    const bool brief = a.b.tokens <= 40 * int64_t(a.b.seqs) || (a.b.tokens <= 80 * int64_t(a.b.seqs) && busy > 1024);
    const bool lengthy = a.b.tokens >= 1500 * int64_t(a.b.seqs);
    if (!brief && busy <= (a.dim <= 64 ? 512 : 256) * (lengthy ? 2 : 1)) {
        // All fit on the chip at once, two to a compute unit or one, or where sequences are long half of them: the second half goes where the shorter ones of the first have been, and 128 rows
        // with all their keys leave a unit alone with one for long.  One head of 64, 14587 tokens: 198 us with 128 rows, 92 with 64 rows and keys dealt to four waves; 8 heads of 128, 2048
        // tokens 40 and 29, 4096 75 and 66; 4 heads, 8000 133 and 100; but 16 heads, 3000 59 and 75, and 32 heads, 1024 25 and 27.  Between
        // one workgroup a place and two: 1500 tokens, 16 heads 32 and 25, 20 heads 32 and 31, two of 1500, 10 heads 32 and 32; but two of 1000, 16 heads 24 and 27, one of 800, 32 heads 20 and 21; with twice
        // the heads of 64 instead 27 and 24, 27 and 27, 28 and 28; 21 and 23, 17 and 18.
        if (a.dim <= 64) narrow_kernel<64, 4><<<small, 512, 0, s>>>(a);
        else narrow_kernel<128, 4><<<small, 512, 0, s>>>(a);
    } else if (a.group % 4 == 0 && !(brief && busy <= 128)) {
        // 60 of up to 200 tokens with 32 heads of 64 on 8 33.8 us with 128 rows of one head, 25.0 with 32 of four; 60 of 96 with heads of 128 44 and 35; 200 of 10 on average 79, with 64 rows
        // of one head 43, 31 with 32 of four; 11 of up to 1500 with heads of 64 61 and 57; one of 16384 2.09 ms both ways.
        // One of 12 with 8 heads of 64 on one 5.2 us, 4.6 with 64 rows of one head
        heads_together(std::integral_constant<int, 4>{});
    } else if (brief) {
        // Sequences that mostly need no more than 64 rows, and no split of their keys, also where two heads share them (200 of 5 with 32 heads of 128 on 16 39 us, 44 with 64 rows of two).
        // 34 of 2 with 32 heads of 128: 19 us with 128 rows, 11 with 64; 8 of 64, which all fit at once, 7.6 and 10; 60 of 96 44 and 45
        if (a.dim <= 64) narrow_kernel<64, 1><<<small, 128, 0, s>>>(a);
        else narrow_kernel<128, 1><<<small, 128, 0, s>>>(a);
    } else if (a.group % 2 == 0) {
        heads_together(std::integral_constant<int, 2>{});
    } else {
        heads_together(std::integral_constant<int, 1>{});
    }
    return hipGetLastError();
}

}  // namespace tl
