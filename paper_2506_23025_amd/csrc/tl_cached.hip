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
// R = max(x + log2 scale_v), so that their fp16 form (2^-11) is exact enough whatever the scales of the blocks are.  The references move only when a score
// is more than 2^8 beyond them, so a tile needs no exchange between lanes.
// Bound: memory.  A sequence's tiles are dealt to the 4 waves of a workgroup, and long ones to several workgroups, in parts whose size
// follows from the whole call's work (read on the device, so that one captured launch serves every length); a second kernel joins them.
#include "tl_attn.hpp"

namespace tl {
namespace {

constexpr int kWaves = 4;
constexpr int kParts = 2048;              // workgroups that a call's work is cut into, about
constexpr int kLeast = 16;                // tiles of a part at least: below this the second kernel costs more than the parts save

constexpr float kInf = __builtin_inff();
constexpr float kSlack = 8.0f;            // log2 of how far a weight may pass its reference (fp16 holds 2^15)

struct Shape {
    int per;                              // tokens of a row tile
    int heads;                            // query heads of a row tile
    int subs;                             // row tiles that the query heads of a key head need
    int rows;                             // per * heads
    int parts;                            // of the call, for one of kv_heads * subs
    int64_t metas;                        // row tiles of the call at most
};

inline Shape shape_of(int64_t seqs, int64_t tokens, bool one, int group, int kv_heads, int nr)
{
    Shape p;
    const int most = 16 * nr;
    p.heads = group < most ? group : most;
    p.subs = (group + p.heads - 1) / p.heads;
    p.per = one ? 1 : most / p.heads;
    p.rows = p.per * p.heads;
    p.parts = kParts / (kv_heads * p.subs);
    if (p.parts < 1) p.parts = 1;
    p.metas = one ? seqs : tokens / p.per + seqs;
    return p;
}

constexpr int kExtra = 4;                 // floats beside a row's sums: m, l, R

// Eight codes as fp16, in order.
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
        // code + 128 in the mantissa of 1024
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

__device__ inline float finite(float x) { return x == -kInf ? 0.0f : x; }
__device__ inline float power(float x) { return __builtin_amdgcn_exp2f(x); }

// Tiles and row tiles of a sequence.
struct Need { int tiles, rts; };
__device__ inline Need need_of(const CachedArgs& a, const Shape& p, int s)
{
    const Span sp = span(a.b, s);
    const int past = cached_of(a.b, s);
    if (sp.n == 0) return {0, 0};
    int64_t len = past < 0 ? 0 : int64_t(past) + sp.n;
    const int64_t room = a.c.pages_per_seq << (a.c.page_shift + 4);
    if (len > room) len = room;
    return {int((len + 63) >> 6), (sp.n + p.per - 1) / p.per};
}

// What a workgroup does: tiles [chunk * size, ...) of row tile rt of sequence seq.
struct Part { int seq, rt, chunk, chunks, size, slot; };

__device__ inline int ceil_div(int a, int b) { return int((unsigned(a) + unsigned(b) - 1u) / unsigned(b)); }

__device__ inline Part find_part(const CachedArgs& a, const Shape& p, int item)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, count = a.b.seqs, per = (count + 63) >> 6;
    float work = 0.0f;
    for (int i = 0; i < per; ++i) {
        const int s = lane * per + i;
        if (s < count) {
            const Need n = need_of(a, p, s);
            work += float(n.tiles) * float(n.rts);
        }
    }
    for (int k = 32; k; k >>= 1) work += __shfl_xor(work, k);
    int size = int(fminf(work * 1.0001f / float(p.parts), 1e9f)) + 1;
    if (size < kLeast) size = kLeast;
    int before = 0, slots = 0;
    while (true) {
        int items = 0, cut = 0;
        for (int i = 0; i < per; ++i) {
            const int s = lo + lane * per + i;
            if (lane * per + i < count) {
                const Need n = need_of(a, p, s);
                const int c = n.tiles ? ceil_div(n.tiles, size) : 1;
                items += n.rts * c;
                if (c > 1) cut += n.rts * c;
            }
        }
        int items_to = items, cut_to = cut;
        for (int k = 1; k < 64; k <<= 1) {
            const int x = __shfl_up(items_to, k), y = __shfl_up(cut_to, k);
            if (lane >= k) { items_to += x; cut_to += y; }
        }
        const uint64_t there = __ballot(before + items_to > item);
        if (!there) return {-1, 0, 0, 0, 0, 0};
        const int owner = __builtin_ctzll(there);
        before += __builtin_amdgcn_readlane(items_to, owner) - __builtin_amdgcn_readlane(items, owner);
        slots += __builtin_amdgcn_readlane(cut_to, owner) - __builtin_amdgcn_readlane(cut, owner);
        lo += owner * per;
        count = count - owner * per < per ? count - owner * per : per;
        if (per == 1) break;
        per = (count + 63) >> 6;
    }
    const Need n = need_of(a, p, lo);
    const int chunks = n.tiles ? ceil_div(n.tiles, size) : 1, i = item - before, rt = i / chunks;
    return {lo, rt, i - rt * chunks, chunks, size, chunks > 1 ? slots + i : -1};
}

// The sums of one row from several parts; `get(i)` gives {m, l, R} of part i.
struct Row { float m, l, R; };

template <bool FP8, int CH, int NR, bool SPLIT>
__global__ __launch_bounds__(64 * kWaves, 2) void cached_kernel(CachedArgs a, Shape p)
{
    constexpr int J = (CH + 3) / 4, DP = CH * 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m16 = lane & 15, g = lane >> 4;
    Part part{int(blockIdx.x), 0, 0, 1, 1 << 30, -1};
    if constexpr (SPLIT) {
        part = find_part(a, p, int(blockIdx.x));
    } else if (a.b.start) {
        const Item it = find_item(a.b, int(blockIdx.x), p.per, 1);
        part.seq = it.seq;
        part.rt = it.i;
    }
    if (part.seq < 0) return;
    const Span sp = span(a.b, part.seq);
    const int past = cached_of(a.b, part.seq);
    const int head = int(blockIdx.y) / p.subs, sub = int(blockIdx.y) - head * p.subs;
    const int first = part.rt * p.per;                    // the row tile's first token in the sequence
    if (first >= sp.n) return;
    const int tokens = sp.n - first < p.per ? sp.n - first : p.per;
    const int heads = a.group - sub * p.heads < p.heads ? a.group - sub * p.heads : p.heads;
    const int rows = tokens * p.heads;                    // those of heads beyond the group are computed and dropped
    const int chunks_dim = a.c.dim >> 4;

    // queries: row r is token r / p.heads, head r % p.heads; positions a row sees
    f16x8 q[NR][J][2];
    int64_t sees[NR];
    int64_t least = int64_t(1) << 40, most = 0;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const int r = n * 16 + m16, t = r / p.heads, h = r - t * p.heads;
        const bool there = r < rows && h < heads;
        sees[n] = past >= 0 ? int64_t(past) + first + (there ? t : 0) + 1 : 0;
        const _Float16* from = a.q.p + int64_t(sp.first + first + (there ? t : 0)) * a.q.token + int64_t(head * a.group + sub * p.heads + (there ? h : 0)) * a.q.head;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = 4 * j + g;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f16x8 x = *reinterpret_cast<const f16x8*>(from + (c < chunks_dim ? c : 0) * 16 + i * 8);
                if (c >= chunks_dim) x = f16x8{0, 0, 0, 0, 0, 0, 0, 0};
                q[n][j][i] = x;
            }
        }
        least = sees[n] < least ? sees[n] : least;
        most = sees[n] > most ? sees[n] : most;
    }
    for (int k = 8; k; k >>= 1) {
        const int64_t x = __shfl_xor(least, k), y = __shfl_xor(most, k);
        least = x < least ? x : least;
        most = y > most ? y : most;
    }
    // tiles of this part that some row sees
    int end = int((most + 63) >> 6);
    {
        const int64_t to = (int64_t(part.chunk) + 1) * part.size;
        if (to < end) end = int(to);
    }
    const int begin = part.chunk * (SPLIT ? part.size : 0);

    f32x4 o[NR][CH];
    float m[NR], l[NR], R[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        m[n] = -kInf;
        R[n] = -kInf;
        l[n] = 0.0f;
#pragma unroll
        for (int d = 0; d < CH; ++d) o[n][d] = f32x4{0, 0, 0, 0};
    }

    const int64_t block_bytes = int64_t(16) * a.c.dim, blocks = int64_t(1) << a.c.page_shift;
    const int in_page = int(blocks - 1);
    auto page_at = [&](int64_t block) { return page_of(a.c, part.seq, block); };
    auto place = [&](int page, int64_t block) { return (int64_t(page < 0 ? 0 : page) * a.c.kv_heads + head) * blocks + (block & in_page); };

    u32x4 kw[4][J], vw[CH];
    float ks = 0.0f, vs = 0.0f;
    int page_k = -1, page_v = -1, next_k = -1, next_v = -1;
    auto load_k = [&](int tile) {
        const uint8_t* from = a.c.k + place(page_k, int64_t(tile) * 4 + (m16 >> 2)) * block_bytes + (m16 & 3) * 16;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int c = 4 * j + g < chunks_dim ? 4 * j + g : 0;
                kw[b][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from + (b * chunks_dim + c) * 64));
            }
    };
    auto load_v = [&](int tile) {
        const int64_t at = place(page_v, int64_t(tile) * 4 + g);
        const uint8_t* from = a.c.v + at * block_bytes + m16 * 16;
#pragma unroll
        for (int d = 0; d < CH; ++d) vw[d] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from + (d < chunks_dim ? d : 0) * 256));
        ks = a.c.ks[at];
        vs = a.c.vs[at];
    };

    int tile = begin + wave;
    if (tile < end) {
        page_k = page_at(int64_t(tile) * 4 + (m16 >> 2));
        page_v = page_at(int64_t(tile) * 4 + g);
        load_k(tile);
        load_v(tile);
        next_k = page_at(int64_t(tile + kWaves) * 4 + (m16 >> 2));
        next_v = page_at(int64_t(tile + kWaves) * 4 + g);
    }
    for (; tile < end; tile += kWaves) {
        const bool more = tile + kWaves < end;
        const bool masked = int64_t(tile) * 64 + 64 > least || !__all(page_v >= 0);
        const bool there = page_v >= 0;
        const float ksc = ks * a.scale, vsc = vs;
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
        if (more) {
            page_k = next_k;
            load_k(tile + kWaves);
        }
        const float lv = __builtin_amdgcn_logf(vsc);
        f16x8 w[NR][2];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            float mx = -kInf;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float x = s[n][b][r] * ksc;
                    if (masked && !(there && int64_t(tile) * 64 + g * 16 + b * 4 + r < sees[n])) x = -kInf;
                    s[n][b][r] = x;
                    mx = fmaxf(mx, x);
                }
            const float top = mx == -kInf ? -kInf : mx + lv;
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
            union { f16x8 v[2]; _Float16 h[16]; } u;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = power(s[n][b][r] - mb);
                    l[n] += x;
                    float y = x * f;
                    if (masked && s[n][b][r] == -kInf) y = 0.0f;
                    u.h[b * 4 + r] = _Float16(y);
                }
            w[n][0] = u.v[0];
            w[n][1] = u.v[1];
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
        if (more) {
            page_v = next_v;
            load_v(tile + kWaves);
            next_k = page_at(int64_t(tile + 2 * kWaves) * 4 + (m16 >> 2));
            next_v = page_at(int64_t(tile + 2 * kWaves) * 4 + g);
        }
    }

    // the four waves' sums of a row
    __shared__ float sums[kWaves][16 * NR][DP + 4];
    __shared__ Row stats[kWaves][16 * NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        l[n] += __shfl_xor(l[n], 16);
        l[n] += __shfl_xor(l[n], 32);
        if (g == 0) stats[wave][n * 16 + m16] = {m[n], l[n], R[n]};
#pragma unroll
        for (int d = 0; d < CH; ++d) *reinterpret_cast<f32x4*>(&sums[wave][n * 16 + m16][d * 16 + g * 4]) = o[n][d];
    }
    __syncthreads();
    constexpr int kQuads = DP / 4;
    float* const to = SPLIT && part.slot >= 0 ? a.part + (int64_t(part.slot) * gridDim.y + blockIdx.y) * p.rows * (DP + kExtra) : nullptr;
    if constexpr (SPLIT) {
        if (part.chunk == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
            int* meta = reinterpret_cast<int*>(a.part + int64_t(2 * p.parts) * gridDim.y * p.rows * (DP + kExtra));
            const int64_t at = a.b.start ? item_base(a.b, part.seq, p.per, 1) + part.rt : part.seq;
            meta[2 * at] = part.slot;
            meta[2 * at + 1] = part.chunks;
        }
    }
    for (int i = threadIdx.x; i < rows * kQuads; i += 64 * kWaves) {
        const int r = i / kQuads, d = (i - r * kQuads) * 4, t = r / p.heads, h = r - t * p.heads;
        if (h >= heads) continue;
        float M = -kInf, top = -kInf, L = 0.0f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            M = fmaxf(M, stats[v][r].m);
            top = fmaxf(top, stats[v][r].R);
        }
        const float Mb = finite(M), Rb = SPLIT && to ? finite(top) : Mb;
        f32x4 sum = {0, 0, 0, 0};
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            L += stats[v][r].l * power(stats[v][r].m - Mb);
            sum += *reinterpret_cast<f32x4*>(&sums[v][r][d]) * power(stats[v][r].R - Rb);
        }
        if (SPLIT && to) {
            float* row = to + r * (DP + kExtra);
            *reinterpret_cast<f32x4*>(row + d) = sum;
            if (d == 0) *reinterpret_cast<f32x4*>(row + DP) = f32x4{M, L, top, 0.0f};
        } else if (d < a.c.dim) {
            sum *= L > 0.0f ? 1.0f / L : L == 0.0f ? 0.0f : L;
            f16x4 y;
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = _Float16(sum[j]);
            *reinterpret_cast<f16x4*>(a.out.p + int64_t(sp.first + first + t) * a.out.token + int64_t(head * a.group + sub * p.heads + h) * a.out.head + d) = y;
        }
    }
}

// Joins the parts of the row tiles that were cut: a wave takes a row, a lane two dimensions.
template <int CH>
__global__ __launch_bounds__(64 * kWaves) void join_kernel(CachedArgs a, Shape p)
{
    constexpr int DP = CH * 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Item it{int(blockIdx.x), 0};
    if (a.b.start) it = find_item(a.b, int(blockIdx.x), p.per, 1);
    if (it.seq < 0) return;
    const Span sp = span(a.b, it.seq);
    const int first = it.i * p.per;
    if (first >= sp.n) return;
    const int* meta = reinterpret_cast<const int*>(a.part + int64_t(2 * p.parts) * gridDim.y * p.rows * (DP + kExtra));
    const int slot = meta[2 * blockIdx.x], chunks = meta[2 * blockIdx.x + 1];
    if (chunks < 2) return;
    const int head = int(blockIdx.y) / p.subs, sub = int(blockIdx.y) - head * p.subs;
    const int tokens = sp.n - first < p.per ? sp.n - first : p.per;
    const int64_t stride = int64_t(gridDim.y) * p.rows * (DP + kExtra);
    for (int r = int(blockIdx.z) * kWaves + wave; r < tokens * p.heads; r += int(gridDim.z) * kWaves) {
        const int t = r / p.heads, h = r - t * p.heads;
        if (sub * p.heads + h >= a.group) continue;
        const float* from = a.part + (int64_t(slot) * gridDim.y + blockIdx.y) * p.rows * (DP + kExtra) + int64_t(r) * (DP + kExtra);
        float M = -kInf;
        for (int c = lane; c < chunks; c += 64) M = fmaxf(M, from[c * stride + DP]);
        for (int k = 32; k; k >>= 1) M = fmaxf(M, __shfl_xor(M, k));
        const float Mb = finite(M);
        float L = 0.0f, x0 = 0.0f, x1 = 0.0f;
        for (int c0 = 0; c0 < chunks; c0 += 64) {
            float w = 0.0f;
            if (c0 + lane < chunks) {
                const f32x4 s = *reinterpret_cast<const f32x4*>(from + (c0 + lane) * stride + DP);
                L += s[1] * power(s[0] - Mb);
                w = power(s[2] - Mb);
            }
            const int n = chunks - c0 < 64 ? chunks - c0 : 64;
            for (int c = 0; c < n; c += 8) {
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const float f = __shfl(w, c + u);        // 0 beyond the last part
                    const float* row = from + (c0 + (c + u < n ? c + u : n - 1)) * stride + (2 * lane < DP ? 2 * lane : 0);
                    x0 += row[0] * f;
                    x1 += row[1] * f;
                }
            }
        }
        for (int k = 32; k; k >>= 1) L += __shfl_xor(L, k);
        const float f = L > 0.0f ? 1.0f / L : L == 0.0f ? 0.0f : L;
        if (2 * lane < a.c.dim)
            *reinterpret_cast<f16x2*>(a.out.p + int64_t(sp.first + first + t) * a.out.token + int64_t(head * a.group + sub * p.heads + h) * a.out.head + 2 * lane) =
                f16x2{_Float16(x0 * f), _Float16(x1 * f)};
    }
}

inline int padded(int64_t dim) { return dim <= 64 ? 64 : 128; }

template <bool FP8, int CH, int NR>
hipError_t launch(const CachedArgs& a, const Shape& p, bool split, hipStream_t s)
{
    const unsigned y = unsigned(a.c.kv_heads * p.subs);
    if (!split) {
        cached_kernel<FP8, CH, NR, false><<<dim3(unsigned(p.metas), y), 64 * kWaves, 0, s>>>(a, p);
        return hipGetLastError();
    }
    cached_kernel<FP8, CH, NR, true><<<dim3(unsigned(p.metas + p.parts), y), 64 * kWaves, 0, s>>>(a, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    join_kernel<CH><<<dim3(unsigned(p.metas), y, unsigned((p.rows + kWaves - 1) / kWaves)), 64 * kWaves, 0, s>>>(a, p);
    return hipGetLastError();
}

}  // namespace

size_t cached_workspace(int64_t seqs, int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t dim)
{
    size_t most = 0;
    for (const bool one : {false, true}) {
        if (one && tokens != seqs) continue;
        const Shape p = shape_of(seqs, tokens, one, int(q_heads / kv_heads), int(kv_heads), 1);
        const size_t n = size_t(2 * p.parts) * size_t(kv_heads * p.subs) * p.rows * (padded(dim) + kExtra) * sizeof(float) + size_t(p.metas) * 2 * sizeof(int);
        if (n > most) most = n;
    }
    return (most + 15) / 16 * 16;
}

hipError_t launch_cached(const CachedArgs& a, int64_t longest, hipStream_t s)
{
    const bool split = longest == 0 || longest > kLeast * 64;
    const Shape p = shape_of(a.b.seqs, a.b.tokens, !a.b.start, a.group, a.c.kv_heads, 1);
    if (a.c.fp8) return padded(a.c.dim) == 64 ? launch<true, 4, 1>(a, p, split, s) : launch<true, 8, 1>(a, p, split, s);
    return padded(a.c.dim) == 64 ? launch<false, 4, 1>(a, p, split, s) : launch<false, 8, 1>(a, p, split, s);
}

}  // namespace tl
