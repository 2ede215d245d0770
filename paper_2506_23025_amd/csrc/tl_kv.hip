// Rotation of queries and keys, and the way of keys and values into the paged 8-bit cache.
//
// A wave takes a block of the cache (16 positions of a sequence) of one head after another, with those of its tokens that the call brings: the tokens of a
// block share a scale, nobody else touches the block, and the cosines and sines of the 16 positions stay in registers for all heads.  A lane has 8
// dimensions (16 bytes) of T consecutive tokens, T = 4, 2 or 1 for heads of up to 128, 64 or 32 dimensions, so that a value's codes of T tokens, neighbours in memory,
// are written together.  Query heads take the same way without the cache.
// Bound: memory for prompts; for a step of a few sequences the chain of dependent reads (length, page, scale).
// Measured: 7 prompts of up to 2048 tokens (6264 in all) with 96 heads of 128 79 us (3.9 TB/s of reads and writes), 92 where pairs are half a head
// apart (the angles of 4 tokens take 64 registers: two waves a SIMD in place of three), the same for both types of codes; one token of 192 sequences with 48 heads 5.1 us; of one sequence 4.0 us.
#include "tl_attn.hpp"

namespace tl {
namespace {

constexpr int kWaves = 4;

template <bool FP8>
__device__ inline float top() { return FP8 ? 448.0f : 127.0f; }

// The codes nearest to four numbers (ties to the even one) that are at most a rounding beyond the top, which every block's scale sees to.
template <bool FP8>
__device__ inline uint32_t four_codes(float a, float b, float c, float d)
{
    if constexpr (FP8) {
        return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true));
    } else {
        // beside 1.5 * 2^23 a whole number's two's complement stands in the last byte
        const float m = 12582912.0f;
        const uint32_t ab = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b + m), __builtin_bit_cast(uint32_t, a + m), 0x0c0c0400u);
        const uint32_t cd = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, d + m), __builtin_bit_cast(uint32_t, c + m), 0x0c0c0400u);
        return ab | cd << 16;
    }
}

template <bool FP8>
__device__ inline uint32_t two_codes(float a, float b) { return four_codes<FP8>(a, b, 0.0f, 0.0f) & 0xffffu; }

// Quotients by one number b, rounded as a division rounds them: with the rounded reciprocal, the remainder of the first guess sets it right (Markstein, IBM
// Journal of Research and Development 34, 1990).  0 for all where b is 0 or NaN.  b is a scale, kSmallest at least and an amax / 127 or / 448: it and its reciprocal
// are ordinary numbers, and so is the remainder of every quotient that is not coded as 0.
struct Divide {
    float b, inv;
    bool any;
    __device__ inline explicit Divide(float x) : b(x), inv(1.0f / x), any(x > 0.0f) {}
    __device__ inline float operator()(float a) const
    {
        const float q = a * inv;
        return any ? __builtin_copysignf(__builtin_fmaf(__builtin_fmaf(-q, b, a), inv, q), a) : 0.0f;      // -0 stays -0
    }
};

template <bool FP8, int I>
__device__ inline float value_of(uint32_t codes)
{
    if constexpr (FP8) return __builtin_amdgcn_cvt_f32_fp8(int(codes), I);
    else return float(int(int8_t(codes >> (8 * I))));
}

template <bool FP8>
__device__ inline uint32_t recode4(uint32_t w, float ratio)
{
    return four_codes<FP8>(value_of<FP8, 0>(w) * ratio, value_of<FP8, 1>(w) * ratio, value_of<FP8, 2>(w) * ratio, value_of<FP8, 3>(w) * ratio);
}

// How 8 dimensions of a lane are turned: not at all; as 4 pairs of neighbours; with the 8 half a head away; one by one (rows of the table or
// halves that are no multiples of 16 bytes).
enum Turn { kNone, kPairs, kHalves, kAny };

// Cosines and sines for 8 dimensions from d on at one position.  pairs: 4 and 4 (c0 and s0); halves: 8 and 8.
struct Angles { f32x4 c0, c1, s0, s1; };

template <Turn TURN>
__device__ inline Angles angles(const Rope r, int64_t pos, int d)
{
    Angles a{};
    if constexpr (TURN == kPairs || TURN == kHalves) {
        const int half = r.rot >> 1, j = TURN == kPairs ? d >> 1 : d < half ? d : d - half;
        const bool there = pos < r.positions;
        const float* t = r.table + (there ? pos : 0) * r.rot + j;
        a.c0 = *reinterpret_cast<const f32x4*>(t);
        a.s0 = *reinterpret_cast<const f32x4*>(t + half);
        if constexpr (TURN == kHalves) {
            a.c1 = *reinterpret_cast<const f32x4*>(t + 4);
            a.s1 = *reinterpret_cast<const f32x4*>(t + half + 4);
        }
        if (!there) {
            const float nan = __builtin_nanf("");
            a.c0 = a.c1 = f32x4{nan, nan, nan, nan};
        }
    }
    return a;
}

// Eight dimensions from d on, in 32 bits, rotated.  `other`: their partners (halves); `row`: where the head begins.
template <Turn TURN>
__device__ inline void turn8(const Rope r, int64_t pos, const _Float16* row, int d, f16x8 own, f16x8 other, const Angles cs, float (&x)[8])
{
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = float(own[i]);
    const int half = r.rot >> 1;
    if (TURN == kNone || d >= r.rot) return;
    if constexpr (TURN == kPairs) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float c = cs.c0[i], s = cs.s0[i], p = x[2 * i], q = x[2 * i + 1];
            const float pc = p * c, qs = q * s, qc = q * c, ps = p * s;
            x[2 * i] = pc - qs;
            x[2 * i + 1] = qc + ps;
        }
    } else if constexpr (TURN == kHalves) {
        const bool second = d >= half;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = x[i] * (i < 4 ? cs.c0[i & 3] : cs.c1[i & 3]), q = float(other[i]) * (i < 4 ? cs.s0[i & 3] : cs.s1[i & 3]);
            x[i] = second ? p + q : p - q;
        }
    } else if constexpr (TURN == kAny) {
        const bool there = pos < r.positions;
        const float* t = r.table + (there ? pos : 0) * r.rot;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = d + i;
            if (e >= r.rot) break;
            const bool second = r.pairs ? (e & 1) : e >= half;
            const int j = r.pairs ? e >> 1 : second ? e - half : e;
            const int o = r.pairs ? e ^ 1 : second ? e - half : e + half;
            const float p = x[i] * t[j], q = float(row[o]) * t[half + j];
            x[i] = !there ? __builtin_nanf("") : second ? p + q : p - q;
        }
    }
}

template <Turn TURN>
__device__ inline f16x8 partners(const Rope r, const _Float16* row, int d)
{
    if constexpr (TURN == kHalves) {
        const int half = r.rot >> 1;
        if (d < r.rot) return *reinterpret_cast<const f16x8*>(row + (d < half ? d + half : d - half));
    }
    return f16x8{0, 0, 0, 0, 0, 0, 0, 0};
}

// What stands in the first `slots` slots of a block, in another scale; lanes i, i + step, ... share it.
template <bool FP8, bool KEY>
__device__ inline void recode(uint8_t* to, int dim, int slots, float ratio, int i, int step)
{
    const int chunks = dim >> 4;
    if constexpr (KEY) {
#pragma clang loop unroll(disable)
        for (; i < slots * chunks; i += step) {
            const int t = i / chunks, c = i - t * chunks;
            uint32_t* w = reinterpret_cast<uint32_t*>(to + ((t >> 2) * chunks + c) * 64 + (t & 3) * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = recode4<FP8>(w[j], ratio);
        }
    } else {
        // whole words of 4 tokens, then the tokens that share a word with new ones
#pragma clang loop unroll(disable)
        for (; i < dim; i += step) {
            uint32_t* w = reinterpret_cast<uint32_t*>(to + i * 16);
            int t = 0;
#pragma clang loop unroll(disable)
            for (; t + 4 <= slots; t += 4) w[t >> 2] = recode4<FP8>(w[t >> 2], ratio);
#pragma clang loop unroll(disable)
            for (; t < slots; ++t) to[i * 16 + t] = uint8_t(two_codes<FP8>(value_of<FP8, 0>(to[i * 16 + t]) * ratio, 0.0f));
        }
    }
}

// The scale of a block that takes tokens with magnitudes up to amax (or an infinity or a NaN: odd) and had `was` (0 if it held nothing).  Rotated keys are coded from
// 32 bits, and a table of tiny numbers could make a scale whose reciprocal is no number, or that is itself so coarse that a magnitude is more than the top of it.
constexpr float kSmallest = 0x1p-80f;
template <bool FP8>
__device__ inline float scale_of(float was, float amax, bool odd)
{
    const float now = fmaxf(was, amax / top<FP8>());
    return odd || !(was == was) ? __builtin_nanf("") : now < kSmallest ? 0.0f : now;
}

// One token's codes of 8 dimensions from d on.
template <bool FP8, bool KEY>
__device__ inline void put_codes(uint8_t* to, int dim, int slot, int d, const float (&x)[8])
{
    if constexpr (KEY) {
        *reinterpret_cast<u32x2*>(to + ((slot >> 2) * (dim >> 4) + (d >> 4)) * 64 + (slot & 3) * 16 + (d & 15)) =
            u32x2{four_codes<FP8>(x[0], x[1], x[2], x[3]), four_codes<FP8>(x[4], x[5], x[6], x[7])};
    } else {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const uint32_t w = two_codes<FP8>(x[i], x[i + 1]);
            to[(d + i) * 16 + slot] = uint8_t(w);
            to[(d + i + 1) * 16 + slot] = uint8_t(w >> 8);
        }
    }
}

__device__ inline void put_row(const Heads& out, int64_t row, int head, int d, const float (&x)[8])
{
    f16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = _Float16(x[i]);
    *reinterpret_cast<f16x8*>(out.p + row * out.token + int64_t(head) * out.head + d) = o;
}

// One token of every sequence: 16 lanes take a head, so a wave four.
template <bool FP8, Turn TURN>
__global__ __launch_bounds__(64 * kWaves) void step_kernel(AppendArgs a)
{
#pragma clang fp contract(off)
    const int seq = blockIdx.x, lane = threadIdx.x & 15, kv = a.kv_heads;
    const int unit = int(blockIdx.y) * (4 * kWaves) + int(threadIdx.x >> 4), d = lane * 8;
    const bool here = d < a.dim && unit < 2 * kv + a.q_heads;
    const bool value = unit >= kv && unit < 2 * kv, key = unit < kv;
    const int head = key ? unit : value ? unit - kv : unit - 2 * kv;
    const int past = same(cached_of(a.b, seq));
    const bool used = past >= 0;
    const Heads in = key ? a.k : value ? a.v : a.q, out = key ? a.k_out : a.q_out;
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (here && used && in.p) {
        const _Float16* row = in.p + int64_t(seq) * in.token + int64_t(head) * in.head;
        const f16x8 own = *reinterpret_cast<const f16x8*>(row + d);
        if (value) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = float(own[i]);
        } else {
            const f16x8 other = partners<TURN>(a.r, row, d);
            Angles cs{};
            if (d < a.r.rot) cs = angles<TURN>(a.r, past, d);
            turn8<TURN>(a.r, past, row, d, own, other, cs, x);
        }
    }
    if (here && !value && out.p) put_row(out, seq, head, d, x);
    // the cache
    const int64_t number = past >> 4;
    const int page = used && a.c.k ? same(page_of(a.c, seq, number)) : -1;
    if (page < 0 || unit >= 2 * kv) return;
    const int slot = past & 15, blocks = 1 << a.c.page_shift;
    const int64_t block = (int64_t(page) * kv + head) * blocks + (number & (blocks - 1));
    float* const scales = key ? a.c.ks : a.c.vs;
    uint8_t* const to = (key ? a.c.k : a.c.v) + block * (int64_t(16) * a.dim);
    const float was = slot ? scales[block] : 0.0f;
    float amax = 0.0f, zero = 0.0f;                          // a NaN or an infinity leaves no 0
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        amax = fmaxf(amax, fabsf(x[i]));
        zero = __builtin_fmaf(x[i], 0.0f, zero);
    }
    for (int s = 8; s; s >>= 1) {
        amax = fmaxf(amax, __shfl_xor(amax, s));
        zero += __shfl_xor(zero, s);
    }
    const float now = scale_of<FP8>(was, amax, !(zero == 0.0f));
    if (lane == 0) scales[block] = now;
    if (slot && now > was) {
        const float ratio = was / now;
        if (key) recode<FP8, true>(to, a.dim, slot, ratio, lane, 16);
        else recode<FP8, false>(to, a.dim, slot, ratio, lane, 16);
    }
    if (!here) return;
    const Divide over(now);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = over(x[i]);
    if (key) put_codes<FP8, true>(to, a.dim, slot, d, x);
    else put_codes<FP8, false>(to, a.dim, slot, d, x);
}

// One block: tokens [0, n) of the call's rows from row0 on, in the block's slots from `slot` on.
struct Place {
    int row0, n, slot;
    int64_t pos;                          // of the block's first slot
};

// What the two ways through a block share: a lane's first slot and dimension, and where a head's rows are.
template <int T>
struct Lane {
    const Rope r;
    const Place at;
    const int dim;
    int lane, first, d;

    __device__ inline Lane(const AppendArgs& a, const Place& place) : r(a.r), at(place), dim(a.dim)
    {
        lane = threadIdx.x & 63;
        first = (lane / (4 * T)) * T;
        d = (lane % (4 * T)) * 8;
    }
    // 8 dimensions of the token in a slot: the head's place in the block's first row is the wave's, what a lane adds to it (15 rows at most) fits 32 bits
    __device__ inline _Float16* place(const Heads h, int head, int slot) const
    {
        char* base = reinterpret_cast<char*>(h.p + int64_t(at.row0) * h.token + int64_t(head) * h.head);
        return reinterpret_cast<_Float16*>(base + (uint32_t(slot - at.slot) * (uint32_t(h.token) * 2u) + uint32_t(d) * 2u));
    }
    __device__ inline void put(const Heads h, int head, int slot, const float (&x)[8]) const
    {
        f16x8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = _Float16(x[i]);
        *reinterpret_cast<f16x8*>(place(h, head, slot)) = o;
    }
    // The block's new scale, written down; what it holds already is coded anew.
    template <bool FP8, bool KEY>
    __device__ inline float rescale(float amax, float zero, int64_t block, uint8_t* to, float* scales) const
    {
        const float was = at.slot ? scales[block] : 0.0f;
        for (int s = 32; s; s >>= 1) amax = fmaxf(amax, __shfl_xor(amax, s));
        const float now = scale_of<FP8>(was, amax, __any(!(zero == 0.0f)));
        if (lane == 0) scales[block] = now;
        if (at.slot && now > was) recode<FP8, KEY>(to, dim, at.slot, was / now, lane, 64);
        return now;
    }
};

// A block that the call fills: every lane has T tokens, and all of them stay in registers.  Of values, T
// neighbours, whose codes are neighbours in memory; of keys and queries those of 16 / T rows that the wave's lanes then read and write side by side.
template <bool FP8, int T, Turn TURN>
struct Whole : Lane<T> {
    const Heads k_out;
    Angles cs[T];
    using Lane<T>::r;
    using Lane<T>::at;
    using Lane<T>::d;
    using Lane<T>::dim;
    using Lane<T>::first;

    template <bool VALUE>
    __device__ inline int slot(int u) const { return VALUE ? first + u : u * (16 / T) + first / T; }

    __device__ inline Whole(const AppendArgs& a, const Place& place) : Lane<T>(a, place), k_out(a.k_out)
    {
        if (d >= dim) d = dim - 8;                           // lanes beyond the head do what its last one does, once more
#pragma unroll
        for (int u = 0; u < T; ++u) {
            cs[u] = Angles{};
            if (d < r.rot) cs[u] = angles<TURN>(r, at.pos + slot<false>(u), d);
        }
    }

    template <bool TURNED>
    __device__ inline void rows(const Heads in, int head, float (&x)[T][8]) const
    {
        f16x8 own[T], other[T];
#pragma unroll
        for (int u = 0; u < T; ++u) {
            const _Float16* p = this->place(in, head, slot<!TURNED>(u));
            own[u] = *reinterpret_cast<const f16x8*>(p);
            if constexpr (TURNED) other[u] = partners<TURN>(r, p - d, d);
        }
#pragma unroll
        for (int u = 0; u < T; ++u) {
            if constexpr (TURNED) {
                turn8<TURN>(r, at.pos + slot<false>(u), this->place(in, head, slot<false>(u)) - d, d, own[u], other[u], cs[u], x[u]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[u][i] = float(own[u][i]);
            }
        }
    }

    __device__ inline void turn(const Heads in, const Heads out, int head) const
    {
        float x[T][8];
        rows<true>(in, head, x);
#pragma unroll
        for (int u = 0; u < T; ++u) this->put(out, head, slot<false>(u), x[u]);
    }

    template <bool KEY>
    __device__ inline void keep(const Heads in, int head, int64_t block, uint8_t* codes, float* scales) const
    {
        float x[T][8];
        rows<KEY>(in, head, x);
        if (KEY && k_out.p) {
#pragma unroll
            for (int u = 0; u < T; ++u) this->put(k_out, head, slot<false>(u), x[u]);
        }
        if (block < 0) return;
        float amax = 0.0f, zero = 0.0f;                      // a NaN or an infinity leaves no 0
#pragma unroll
        for (int u = 0; u < T; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                amax = fmaxf(amax, fabsf(x[u][i]));
                zero = __builtin_fmaf(x[u][i], 0.0f, zero);
            }
        uint8_t* const to = codes + block * (int64_t(16) * dim);
        const Divide over(this->template rescale<FP8, KEY>(amax, zero, block, to, scales));
        if constexpr (!KEY && T > 1) {                       // the codes of a lane's tokens are neighbours
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint8_t* p = to + (d + i) * 16 + first;
                if constexpr (T == 4) *reinterpret_cast<uint32_t*>(p) = four_codes<FP8>(over(x[0][i]), over(x[1][i]), over(x[2][i]), over(x[3][i]));
                if constexpr (T == 2) *reinterpret_cast<uint16_t*>(p) = uint16_t(two_codes<FP8>(over(x[0][i]), over(x[1][i])));
            }
        } else {
#pragma unroll
            for (int u = 0; u < T; ++u) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[u][i] = over(x[u][i]);
                put_codes<FP8, KEY>(to, dim, slot<!KEY>(u), d, x[u]);
            }
        }
    }
};

// Any other block: 16 / T tokens at a time, and once more when the scale is known.
template <bool FP8, int T, Turn TURN>
struct Some : Lane<T> {
    const Heads k_out;
    using Lane<T>::r;
    using Lane<T>::at;
    using Lane<T>::d;
    using Lane<T>::dim;
    using Lane<T>::first;

    __device__ inline Some(const AppendArgs& a, const Place& place) : Lane<T>(a, place), k_out(a.k_out) {}
    __device__ inline int slot(int u) const { return u * (16 / T) + first / T; }
    __device__ inline bool has(int u) const { return d < dim && slot(u) >= at.slot && slot(u) < at.slot + at.n; }

    template <bool TURNED>
    __device__ inline void row(const Heads in, int head, int u, float (&x)[8]) const
    {
        const _Float16* p = this->place(in, head, slot(u));
        const f16x8 own = *reinterpret_cast<const f16x8*>(p);
        if constexpr (TURNED) {
            Angles cs{};
            if (d < r.rot) cs = angles<TURN>(r, at.pos + slot(u), d);
            turn8<TURN>(r, at.pos + slot(u), p - d, d, own, partners<TURN>(r, p - d, d), cs, x);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = float(own[i]);
        }
    }

    // rotated rows, or zeros where the sequence is not in use
    __device__ inline void turn(const Heads in, const Heads out, int head, bool used) const
    {
#pragma clang loop unroll(disable)
        for (int u = at.slot / (16 / T); u * (16 / T) < at.slot + at.n; ++u) {
            if (!has(u)) continue;
            float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (used) row<true>(in, head, u, x);
            this->put(out, head, slot(u), x);
        }
    }

    template <bool KEY>
    __device__ inline void keep(const Heads in, int head, int64_t block, uint8_t* codes, float* scales) const
    {
        float amax = 0.0f, zero = 0.0f;                      // a NaN or an infinity leaves no 0
#pragma clang loop unroll(disable)
        for (int u = at.slot / (16 / T); u * (16 / T) < at.slot + at.n; ++u) {
            if (!has(u)) continue;
            float x[8];
            row<KEY>(in, head, u, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                amax = fmaxf(amax, fabsf(x[i]));
                zero = __builtin_fmaf(x[i], 0.0f, zero);
            }
        }
        uint8_t* const to = codes + block * (int64_t(16) * dim);
        const Divide over(block < 0 ? 0.0f : this->template rescale<FP8, KEY>(amax, zero, block, to, scales));
#pragma clang loop unroll(disable)
        for (int u = at.slot / (16 / T); u * (16 / T) < at.slot + at.n; ++u) {
            if (!has(u)) continue;
            float x[8];
            row<KEY>(in, head, u, x);
            if (KEY && k_out.p) this->put(k_out, head, slot(u), x);        // which may be the row that was read
            if (block < 0) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = over(x[i]);
            put_codes<FP8, KEY>(to, dim, slot(u), d, x);
        }
    }
};

template <bool FP8, int T, Turn TURN, bool WHOLE>
__global__ __launch_bounds__(64 * kWaves) void append_kernel(AppendArgs a, int each)
{
    Item it{int(blockIdx.x), 0};
    if (a.b.start) it = find_item(a.b, int(blockIdx.x), 16, 2);
    it = {same(it.seq), same(it.i)};
    if (it.seq < 0) return;
    Span sp = span(a.b, it.seq);
    sp = {same(sp.first), same(sp.n)};
    const int past = same(cached_of(a.b, it.seq));
    const bool used = past >= 0;
    const int before = used ? past : 0;
    // tokens [i0, i1) of the sequence are those of this block
    const int64_t number = int64_t(before >> 4) + it.i;
    const int64_t i0 = it.i == 0 ? 0 : number * 16 - before;
    const int64_t i1 = number * 16 + 16 - before < sp.n ? number * 16 + 16 - before : sp.n;
    if (i0 >= i1) return;
    const Place at{sp.first + int(i0), int(i1 - i0), int((before + i0) & 15), number * 16};
    const int units = 2 * a.kv_heads + a.q_heads;
    int unit = int(blockIdx.y) * kWaves * each + same(threadIdx.x >> 6);
    const int stop = unit + kWaves * each < units ? unit + kWaves * each : units;
    if (unit >= stop) return;
    // a wave's heads: keys, values, queries
    const int kv = a.kv_heads, blocks = 1 << a.c.page_shift;
    const int page = used && a.c.k ? same(page_of(a.c, it.seq, number)) : -1;
    auto place = [&](int head) { return page < 0 ? int64_t(-1) : (int64_t(page) * kv + head) * blocks + (number & (blocks - 1)); };
    if (WHOLE && at.n == 16 && used) {
        const Whole<FP8, T, TURN> work(a, at);
        for (; unit < stop; unit += kWaves) {
            if (unit >= 2 * kv) work.turn(a.q, a.q_out, unit - 2 * kv);
            else if (unit < kv) work.template keep<true>(a.k, unit, place(unit), a.c.k, a.c.ks);
            else if (page >= 0) work.template keep<false>(a.v, unit - kv, place(unit - kv), a.c.v, a.c.vs);
        }
    } else {
        const Some<FP8, T, TURN> work(a, at);
        for (; unit < stop; unit += kWaves) {
            if (unit >= 2 * kv) work.turn(a.q, a.q_out, unit - 2 * kv, used);
            else if (unit >= kv) { if (page >= 0) work.template keep<false>(a.v, unit - kv, place(unit - kv), a.c.v, a.c.vs); }
            else if (used) work.template keep<true>(a.k, unit, place(unit), a.c.k, a.c.ks);
            else if (a.k_out.p) work.turn(a.k, a.k_out, unit, false);
        }
    }
}

template <bool FP8, int T, Turn TURN>
hipError_t launch(const AppendArgs& a, hipStream_t s)
{
    const int units = 2 * a.kv_heads + a.q_heads;
    if (!a.b.start) {
        step_kernel<FP8, TURN><<<dim3(unsigned(a.b.seqs), unsigned((units + 4 * kWaves - 1) / (4 * kWaves))), 64 * kWaves, 0, s>>>(a);
        return hipGetLastError();
    }
    const int64_t items = a.b.tokens / 16 + 2 * int64_t(a.b.seqs);
    // heads for each wave, as many as leave the chip 16 waves for each SIMD (8: 86 us for 81, 32: 91, at 6264 tokens of 96 heads)
    int64_t each = items * units / (16 * 1024);
    if (each < 1) each = 1;
    if (each > (units + kWaves - 1) / kWaves) each = (units + kWaves - 1) / kWaves;
    const dim3 grid(unsigned(items), unsigned((units + kWaves * each - 1) / (kWaves * each)));
    // Sequences of a few tokens have few whole blocks, and what fills those at a time has twice to four times the registers: 234 of 3 tokens on average with 40 heads of 96 in all 26 us
    // with it, 15.5 without; 100 of 16 with 32 heads of 128 18.8 and 18.6; one of 1000 with 48 heads 10.9 with it.  With a table of an odd width it takes all of a SIMD's:
    // 5000 tokens of 48 heads 115 and 68.
    if (TURN == kAny || a.b.tokens < 16 * int64_t(a.b.seqs)) append_kernel<FP8, T, TURN, false><<<grid, 64 * kWaves, 0, s>>>(a, int(each));
    else append_kernel<FP8, T, TURN == kAny ? kNone : TURN, true><<<grid, 64 * kWaves, 0, s>>>(a, int(each));
    return hipGetLastError();
}

template <bool FP8, Turn TURN>
hipError_t launch_dim(const AppendArgs& a, hipStream_t s)
{
    return a.dim <= 32 ? launch<FP8, 1, TURN>(a, s) : a.dim <= 64 ? launch<FP8, 2, TURN>(a, s) : launch<FP8, 4, TURN>(a, s);
}

template <bool FP8>
hipError_t launch_turn(const AppendArgs& a, hipStream_t s)
{
    if (!a.r.table) return launch_dim<FP8, kNone>(a, s);
    if (!a.r.wide) return launch_dim<FP8, kAny>(a, s);
    return a.r.pairs ? launch_dim<FP8, kPairs>(a, s) : launch_dim<FP8, kHalves>(a, s);
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, hipStream_t s) { return a.c.fp8 ? launch_turn<true>(a, s) : launch_turn<false>(a, s); }

}  // namespace tl
