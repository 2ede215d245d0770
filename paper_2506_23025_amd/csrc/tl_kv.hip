// Rotation of queries and keys, and the way of keys and values into the paged 8-bit cache.
//
// A wave takes up to 16 tokens of one head, those of one call that fall into one block of the cache (positions 16 b .. 16 b + 15 of a sequence),
// since they share a scale: the tokens' values stay in its registers (8 dimensions a lane, so dim / 8 lanes to a token), the largest magnitude is
// a reduction over the wave, and nobody else touches the block.  Query heads take the same way without the cache.
// Bound: memory for prompts; for a step of a few sequences the chain of dependent reads (length, page, scale).
#include "tl_attn.hpp"

namespace tl {
namespace {

constexpr int kWaves = 4;

template <bool FP8>
__device__ inline float top() { return FP8 ? 448.0f : 127.0f; }

// The nearest code of x, |x| at most a rounding beyond the top; NaN has none and gives anything.
template <bool FP8>
__device__ inline uint32_t code_of(float x)
{
    x = fminf(fmaxf(x, -top<FP8>()), top<FP8>());
    if constexpr (FP8) return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false)) & 255u;
    else return uint32_t(int(rintf(x))) & 255u;
}

template <bool FP8>
__device__ inline float value_of(uint32_t code)
{
    if constexpr (FP8) return __builtin_amdgcn_cvt_f32_fp8(int(code), 0);
    else return float(int(int8_t(code)));
}

template <bool FP8>
__device__ inline uint32_t recode4(uint32_t w, float ratio)
{
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) r |= code_of<FP8>(value_of<FP8>((w >> (8 * i)) & 255u) * ratio) << (8 * i);
    return r;
}

// Dimensions d .. d + 7 of one token's head, rotated.  `row` is where the head begins.
__device__ inline void rotated(const Rope& r, const _Float16* row, int d, int64_t pos, float (&x)[8])
{
#pragma clang fp contract(off)
    const f16x8 own = *reinterpret_cast<const f16x8*>(row + d);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = float(own[i]);
    if (!r.table || d >= r.rot) return;
    const int half = r.rot >> 1;
    if (pos >= r.positions) {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (d + i < r.rot) x[i] = __builtin_nanf("");
        return;
    }
    const float* cs = r.table + pos * r.rot;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = d + i;
        if (e >= r.rot) break;
        const bool second = r.pairs ? (e & 1) : e >= half;
        const int j = r.pairs ? e >> 1 : second ? e - half : e;
        const int other = r.pairs ? e ^ 1 : second ? e - half : e + half;
        const float c = cs[j], s = cs[half + j], y = float(row[other]);
        const float p = x[i] * c, q = y * s;
        x[i] = second ? p + q : p - q;
    }
}

// One head of the block: `n` tokens in the slots from `slot` on, of whom token i stands in row `row0 + i`.
template <bool FP8, bool KEY>
__device__ inline void put_block(const AppendArgs& a, const Heads& in, int head, int row0, int n, int slot, int64_t pos, int page, int blk,
                                 uint8_t* codes, float* scales)
{
#pragma clang fp contract(off)
    const int lane = threadIdx.x & 63, per = a.dim >> 3, at_once = 64 / per;
    const int t_lane = lane / per, d = (lane - t_lane * per) * 8;
    float x[4][8];
    float amax = 0.0f;
    bool odd = false;                                    // a NaN or an infinity
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int t = u * at_once + t_lane;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[u][i] = 0.0f;
        if (t_lane >= at_once || t >= n) continue;
        const _Float16* row = in.p + int64_t(row0 + t) * in.token + int64_t(head) * in.head;
        if constexpr (KEY) {
            rotated(a.r, row, d, pos + t, x[u]);
            if (a.k_out.p) {
                f16x8 o;
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = _Float16(x[u][i]);
                *reinterpret_cast<f16x8*>(a.k_out.p + int64_t(row0 + t) * a.k_out.token + int64_t(head) * a.k_out.head + d) = o;
            }
        } else {
            const f16x8 own = *reinterpret_cast<const f16x8*>(row + d);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] = float(own[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            amax = fmaxf(amax, fabsf(x[u][i]));
            odd |= !(fabsf(x[u][i]) < __builtin_inff());
        }
    }
    if (page < 0) return;
    for (int s = 32; s; s >>= 1) amax = fmaxf(amax, __shfl_xor(amax, s));
    odd = __any(odd);
    const int blocks = 1 << a.c.page_shift, chunks = a.dim >> 4;
    const int64_t block = (int64_t(page) * a.kv_heads + head) * blocks + blk;
    uint8_t* const to = codes + block * (int64_t(16) * a.dim);
    const float was = slot ? scales[block] : 0.0f;
    float now = fmaxf(was, amax / top<FP8>());
    if (odd || !(was == was)) now = __builtin_nanf("");
    if (lane == 0) scales[block] = now;
    if (slot && now > was) {                             // what stands before the new tokens, in the new scale
        const float ratio = was / now;
        if constexpr (KEY) {
            // 4 tokens of 16 dimensions are 64 bytes: one lane, one token
            for (int i = lane; i < slot * chunks; i += 64) {
                const int t = i / chunks, c = i - t * chunks;
                uint32_t* w = reinterpret_cast<uint32_t*>(to + ((t >> 2) * chunks + c) * 64 + (t & 3) * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = recode4<FP8>(w[j], ratio);
            }
        } else {
            for (int i = lane; i < a.dim; i += 64) {
                for (int t = 0; t < slot; ++t) to[i * 16 + t] = uint8_t(code_of<FP8>(value_of<FP8>(to[i * 16 + t]) * ratio));
            }
        }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int t = u * at_once + t_lane;
        if (t_lane >= at_once || t >= n) continue;
        const int at = slot + t;
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i >> 2] |= (now > 0.0f ? code_of<FP8>(x[u][i] / now) : 0u) << (8 * (i & 3));
        if constexpr (KEY) {
            *reinterpret_cast<u32x2*>(to + ((at >> 2) * chunks + (d >> 4)) * 64 + (at & 3) * 16 + (d & 15)) = u32x2{w[0], w[1]};
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) to[(d + i) * 16 + at] = uint8_t(w[i >> 2] >> (8 * (i & 3)));
        }
    }
}

__device__ inline void turn_head(const AppendArgs& a, const Heads& in, const Heads& out, int head, int row0, int n, int64_t pos, bool used)
{
    const int lane = threadIdx.x & 63, per = a.dim >> 3, at_once = 64 / per;
    const int t_lane = lane / per, d = (lane - t_lane * per) * 8;
    if (t_lane >= at_once) return;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int t = u * at_once + t_lane;
        if (t >= n) break;
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (used) rotated(a.r, in.p + int64_t(row0 + t) * in.token + int64_t(head) * in.head, d, pos + t, x);
        f16x8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = _Float16(x[i]);
        *reinterpret_cast<f16x8*>(out.p + int64_t(row0 + t) * out.token + int64_t(head) * out.head + d) = o;
    }
}

template <bool FP8>
__global__ __launch_bounds__(64 * kWaves) void append_kernel(AppendArgs a)
{
    Item it{int(blockIdx.x), 0};
    if (a.b.start) it = find_item(a.b, int(blockIdx.x), 16, 2);
    if (it.seq < 0) return;
    const Span sp = span(a.b, it.seq);
    const int past = cached_of(a.b, it.seq);
    const bool used = past >= 0;
    const int before = used ? past : 0;
    // tokens [i0, i1) of the sequence are those of this block
    const int64_t block = (before >> 4) + it.i;
    const int i0 = it.i == 0 ? 0 : int(block * 16 - before);
    const int i1 = block * 16 + 16 - before < sp.n ? int(block * 16 + 16 - before) : sp.n;
    if (i0 >= i1) return;
    const int n = i1 - i0, row0 = sp.first + i0;
    const int64_t pos = int64_t(before) + i0;
    int unit = int(blockIdx.y) * kWaves + int(threadIdx.x >> 6);
    const int kv = a.kv_heads;
    if (unit < 2 * kv) {
        const bool key = unit < kv;
        const int head = key ? unit : unit - kv;
        if (!used || !a.c.k) {
            if (key && a.k_out.p) turn_head(a, a.k, a.k_out, head, row0, n, pos, used);
            return;
        }
        const int page = page_of(a.c, it.seq, block), blk = int(block & ((1 << a.c.page_shift) - 1));
        if (key) put_block<FP8, true>(a, a.k, head, row0, n, int(pos & 15), pos, page, blk, a.c.k, a.c.ks);
        else put_block<FP8, false>(a, a.v, head, row0, n, int(pos & 15), pos, page, blk, a.c.v, a.c.vs);
        return;
    }
    unit -= 2 * kv;
    if (unit < a.q_heads && a.q_out.p) turn_head(a, a.q, a.q_out, unit, row0, n, pos, used);
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, hipStream_t s)
{
    const int64_t items = a.b.start ? a.b.tokens / 16 + 2 * int64_t(a.b.seqs) : a.b.seqs;
    const int units = 2 * a.kv_heads + a.q_heads;
    const dim3 grid(unsigned(items), unsigned((units + kWaves - 1) / kWaves));
    if (a.c.fp8) append_kernel<true><<<grid, 64 * kWaves, 0, s>>>(a);
    else append_kernel<false><<<grid, 64 * kWaves, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace tl
