// The residual's addition with the norm, the gate, and rows as they are, into fp16 and 8 bits.
#include "tl_rows.hpp"

namespace tl {
namespace {

// The value of the lane that DPP control CTRL names; 0 where there is none.
template <int CTRL, int ROWS>
__device__ inline uint32_t moved(uint32_t x) { return uint32_t(__builtin_amdgcn_update_dpp(0, int(x), CTRL, ROWS, 15, true)); }
template <int CTRL, int ROWS>
__device__ inline double moved(double x)
{
    const u32x2 u = __builtin_bit_cast(u32x2, x);
    return __builtin_bit_cast(double, u32x2{moved<CTRL, ROWS>(u[0]), moved<CTRL, ROWS>(u[1])});
}

// Over the wave, the result in all lanes: from the lane 1, 2, 4 and 8 before in the row of 16, a row's last lane to the next row, lane 31 to rows 2 and 3.
template <class T, class F>
__device__ inline T over_wave(T x, F f)
{
    x = f(x, moved<0x111, 15>(x));
    x = f(x, moved<0x112, 15>(x));
    x = f(x, moved<0x114, 15>(x));
    x = f(x, moved<0x118, 15>(x));
    x = f(x, moved<0x142, 10>(x));
    return f(x, moved<0x143, 12>(x));
}
__device__ inline double wave_sum(double x)
{
    const u32x2 u = __builtin_bit_cast(u32x2, over_wave(x, [](double a, double b) { return a + b; }));
    return __builtin_bit_cast(double, u32x2{uint32_t(__builtin_amdgcn_readlane(int(u[0]), 63)), uint32_t(__builtin_amdgcn_readlane(int(u[1]), 63))});
}
__device__ inline uint32_t wave_max(uint32_t x)
{
    return uint32_t(__builtin_amdgcn_readlane(int(over_wave(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; })), 63));
}

// g / (1 + e^-g) * u in fp64; an infinity or NaN where g or u is not finite.  e^-g = 2^n e^r with |r| <= log(2) / 2;
// e^r by the polynomial of degree 10 that agrees with it at the eleven nodes of Chebyshev's on that interval (off by 2^-51); the quotient from the hardware's reciprocal q of d = 1 + e^-g, which is off by e = 1 - d q, as
// w q (1 + e + e^2).  A product in fp64 costs what one in fp32 does here; conversions cost more, so n is found by a sum that leaves it in the lowest bits, and 2^n goes into the exponent by an
// integer addition.
// How far it is off: 2^-51 of itself for g > -1, 2^-50.1 down to -10, 2^-49.5 to -22, 2^-48.9 to -40, 2^-47.8 at -104, below which fp32 has nothing: log(2) is one number, and what it lacks moves e^-g by n 2^-55.2.  Two numbers for it,
// one more sum a value, would keep 2^-50.7 and change no result: over every g of fp16 and every mantissa of u (72 million pairs) both give the exact value's rounding to fp32 but for the same 100 pairs,
// all with |g| <= 2^-16, where g / 2 + g^2 / 4 is a tie between two numbers and what decides is below 2^-53 of it.
struct Gate {
    // in scalar registers: the compiler would move each into the sum's registers first
    double c[10] = {0x1.28a2ca617b969p-22, 0x1.72fafebdaf273p-19, 0x1.a019a6611cad5p-16, 0x1.a01978b8b3d18p-13, 0x1.6c16c17f46982p-10,
                    0x1.1111112ddae8bp-7, 0x1.55555555520a4p-5, 0x1.555555554b736p-3, 0x1.0000000000005p-1, 0x1.000000000001ep+0};
    double rate = -0x1.71547652b82fep+0, log2 = -0x1.62e42fefa39efp-1, shift = 0x1.8p52;
    __device__ Gate()
    {
#pragma unroll
        for (int i = 1; i < 10; ++i) asm("" : "+s"(c[i]));
        asm("" : "+s"(rate), "+s"(log2), "+v"(shift), "+v"(c[0]));
    }
    __device__ inline float operator()(float g, float u) const
    {
        const double x = double(__builtin_amdgcn_fmed3f(g, -700.0f, 700.0f));
        const double z = __builtin_fma(x, rate, shift), n = z - shift;
        const double r = __builtin_fma(n, log2, -x);      // log(2) rounded moves it by n 2^-55
        double p = __builtin_fma(c[0], r, c[1]);
#pragma unroll
        for (int i = 2; i < 10; ++i) p = __builtin_fma(p, r, c[i]);
        p = __builtin_fma(p, r, 1.0);
        u32x2 t = __builtin_bit_cast(u32x2, p);
        t[1] += __builtin_bit_cast(u32x2, z)[0] << 20;    // |n| <= 1010: within the exponent's range
        const double d = 1.0 + __builtin_bit_cast(double, t), q = __builtin_amdgcn_rcp(d);
        const double e = __builtin_fma(-d, q, 1.0), w = double(g * u) * q;      // g * u is exact: 22 bits
        return float(__builtin_fma(w, __builtin_fma(e, e, e), w));
    }
};

// Eight values from place d of a row on; 0 behind its end.
__device__ inline void take(const _Float16* row, int d, int dim, float* v)
{
    if (d + 8 <= dim) {
        const f16x8 x = *reinterpret_cast<const f16x8*>(row + d);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = float(x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = d + i < dim ? float(row[d + i]) : 0.0f;
    }
}
__device__ inline void take(const float* row, int d, int dim, float* v)
{
    if (d + 8 <= dim) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(row + d), y = *reinterpret_cast<const f32x4*>(row + d + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = x[i], v[4 + i] = y[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = d + i < dim ? row[d + i] : 0.0f;
    }
}
__device__ inline void put(_Float16* row, int d, int dim, const float* v)
{
    if (d + 8 <= dim) {
        f16x8 x;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = _Float16(rounded(v[i]));
        *reinterpret_cast<f16x8*>(row + d) = x;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d + i < dim) row[d + i] = _Float16(rounded(v[i]));
    }
}
__device__ inline void put(float* row, int d, int dim, const float* v)
{
    if (d + 8 <= dim) {
        *reinterpret_cast<f32x4*>(row + d) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4*>(row + d + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d + i < dim) row[d + i] = v[i];
    }
}

// W waves hold a row in registers, C pieces of 8 values a lane; workgroups of four rows where a wave has one to itself.  One pass over memory: a row is read once, its sum of squares (fp64: squares of
// fp32 numbers are exact there, and with the root and the quotient in it too every rounding falls as the formula's does, whatever the order) and its largest magnitude go over the wave by DPP and over
// the waves through LDS.  What bounds it (MI355X): a lone row the launch, 2.4 us; the norm memory, 8192 rows of 4096 places with a residual in fp16 to 8 bits 45 us = 5.2 TB/s read and written, what a
// large copy reaches on the card; 32-bit residuals 5.4 TB/s.  The gate the vector unit, busy 77 % of the time at 4096 rows of 11008 (26.2 M instructions, fp64 conversions and reciprocals longer than others), 62 to 65 us = 3.5 TB/s:
// 37 instructions a value, 21 of them in fp64.  Before the polynomial of degree 10, constants in scalar registers, conversions and selects taken out it took 116 us.
// What it waits for besides: a piece is loaded behind a branch and converted in it, so each load is waited for before the next is asked for; x, residual and weight are three trips to memory one after the other
// (192 rows of 4096 with a 32-bit residual 4.0 us, a lone row 2.4).  The last piece of a row that is no multiple of 8 is loaded a value at a time: 8192 rows of 4093 places 68 us in a loop that takes 48 for 4096, the gate of 4096 rows of
// 11005 73 and 68.  The gate of rows of more than 32768 places (16 waves, 8 pieces) keeps 75 registers in memory: 256 rows of 65536 27.7 us, of 32768 15.8.
template <RowsKind KIND, int W, int C>
__global__ void __launch_bounds__(W == 1 ? 256 : 64 * W) rows_kernel(RowsArgs a)
{
    constexpr bool NORM = KIND >= kNormRows;
    __shared__ double sums[W];
    __shared__ uint32_t tops[W];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = W == 1 ? int64_t(blockIdx.x) * 4 + wave : blockIdx.x;
    if (W == 1 && row >= a.rows) return;
    const int first = (W == 1 ? lane : int(threadIdx.x)) * 8;
    const int wave_first = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave) * 512;
    constexpr int STEP = 64 * 8 * W;
    const int dim = a.dim;
    const _Float16* const xa = static_cast<const _Float16*>(a.a.p) + row * a.a.stride;
    float v[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) take(xa, first + c * STEP, dim, v[c]);
    if constexpr (KIND == kGatedRows) {
        const _Float16* const xg = static_cast<const _Float16*>(a.b.p) + row * a.b.stride;
        const Gate gated;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (wave_first + c * STEP >= dim) break;      // the pieces that a wave has none of
            float g[8];
            take(xg, first + c * STEP, dim, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = gated(g[i], v[c][i]);
        }
    }
    if constexpr (NORM) {
        if constexpr (KIND == kNormSum16) {
            const _Float16* const xr = static_cast<const _Float16*>(a.b.p) + row * a.b.stride;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float r[8];
                take(xr, first + c * STEP, dim, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = float(_Float16(rounded(r[i] + v[c][i])));
                if (a.sum.p) put(static_cast<_Float16*>(a.sum.p) + row * a.sum.stride, first + c * STEP, dim, v[c]);
            }
        }
        if constexpr (KIND == kNormSum32) {
            const float* const xr = static_cast<const float*>(a.b.p) + row * a.b.stride;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float r[8];
                take(xr, first + c * STEP, dim, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = r[i] + v[c][i];
                if (a.sum.p) put(static_cast<float*>(a.sum.p) + row * a.sum.stride, first + c * STEP, dim, v[c]);
            }
        }
        double ss = 0.0;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = __builtin_fma(double(v[c][i]), double(v[c][i]), ss);
        ss = wave_sum(ss);
        if constexpr (W > 1) {
            if (lane == 0) sums[wave] = ss;
            __syncthreads();
            ss = 0.0;
#pragma unroll
            for (int w = 0; w < W; ++w) ss += sums[w];
        }
        const float r = float(1.0 / sqrt(ss / double(dim) + a.eps));
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] *= r;
            if (a.weight) {
                float w[8];
                take(a.weight, first + c * STEP, dim, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] *= w[i];
            }
        }
    }
    // The largest magnitude as its bits: they order as the numbers do, infinities and NaN above all.  Places behind the row are 0, or NaN in a row that is.
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t u = __builtin_bit_cast(uint32_t, v[c][i]) & 0x7fffffffu;
            top = u > top ? u : top;
        }
    if constexpr (KIND == kGatedRows) {
        // what is not finite in y: the product, but for a gate of -infinity, which has none
        if (a.y.p && __any(top >= 0x7f800000u)) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float g[8], u[8];
                take(static_cast<const _Float16*>(a.b.p) + row * a.b.stride, first + c * STEP, dim, g);
                take(xa, first + c * STEP, dim, u);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (!__builtin_isfinite(g[i] * u[i])) v[c][i] = g[i] == -__builtin_inff() ? __builtin_nanf("") : g[i] * u[i];
            }
        }
    }
    if (a.y.p) {
#pragma unroll
        for (int c = 0; c < C; ++c) put(static_cast<_Float16*>(a.y.p) + row * a.y.stride, first + c * STEP, dim, v[c]);
    }
    if (!a.out.codes) return;
    top = wave_max(top);
    if constexpr (W > 1) {
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        top = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) top = tops[w] > top ? tops[w] : top;
    }
    const float most = __builtin_bit_cast(float, top);
    const bool finite = top < 0x7f800000u, some = finite && most >= 0x1p-100f;
    const float inverse = some ? 127.0f / most : 0.0f;
    if (first == 0) a.out.scales[row] = some ? most / 127.0f : finite ? 0.0f : __builtin_nanf("");
    int8_t* const codes = a.out.codes + row * a.out.stride;
    const bool odd = lane & 1;
    const uint32_t keep = some ? ~0u : 0u;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        // A product below 2^22 is rounded to a whole number by a sum that leaves it in the lowest bits.
        uint32_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = __builtin_bit_cast(uint32_t, rounded(v[c][i] * inverse) + 0x1.8p23f);
        // Two lanes hold a block of 16.  Each has two bytes of all four words of it (places s and 4 + s of its half); the even lane writes the first two words, the odd lane the others.
        const auto bytes = [&](int i, int j, int k, int l) {
            return __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[l], q[k], 0x0C0C0400u), __builtin_amdgcn_perm(q[j], q[i], 0x0C0C0400u), 0x05040100u) & keep;
        };
        const uint32_t lo = bytes(0, 4, 1, 5), hi = bytes(2, 6, 3, 7);
        const uint32_t got = moved<0xB1, 15>(odd ? lo : hi), own = odd ? hi : lo;
        const uint32_t l = odd ? got : own, h = odd ? own : got;
        const int d = first + c * STEP;
        if ((d & ~15) < dim) *reinterpret_cast<u32x2*>(codes + d) = u32x2{(l & 0xffffu) | h << 16, l >> 16 | (h & 0xffff0000u)};
    }
}

template <RowsKind KIND, int W, int C>
hipError_t launch(const RowsArgs& a, hipStream_t s)
{
    const unsigned groups = W == 1 ? unsigned((a.rows + 3) / 4) : unsigned(a.rows);
    hipLaunchKernelGGL((rows_kernel<KIND, W, C>), dim3(groups), dim3(W == 1 ? 256 : 64 * W), 0, s, a);
    return hipGetLastError();
}

template <RowsKind KIND>
hipError_t launch_kind(const RowsArgs& a, hipStream_t s)
{
    // A piece a lane as long as 16 waves hold the row; longer rows, where there are many, 8 waves with more.  Measured (us): 192 rows of 4096 places with a residual in fp16, 4 / 8 / 16
    // waves 4.6 / 4.0 / 4.5; 2048 of 2048, 1 / 4 / 8 waves 11.3 / 10.0 / 11.4; 600 of 8192, 8 / 16 waves 11.1 / 13.0; 4096 of 11008, 8 / 12 / 16 waves 65 / 70 / 71, 64 rows of it 6.7 / 6.0 / 6.1.
    const int pieces = (a.dim + 7) / 8;
    const bool many = a.rows >= 256;
    if (pieces <= 64) return launch<KIND, 1, 1>(a, s);
    if (pieces <= 128) return launch<KIND, 2, 1>(a, s);
    if (pieces <= 256) return launch<KIND, 4, 1>(a, s);
    if (pieces <= 384) return launch<KIND, 6, 1>(a, s);
    if (pieces <= 512) return launch<KIND, 8, 1>(a, s);
    if (pieces <= 1024) return many ? launch<KIND, 8, 2>(a, s) : launch<KIND, 16, 1>(a, s);
    if (pieces <= 1536 && many) return launch<KIND, 8, 3>(a, s);
    if (pieces <= 2048) return many ? launch<KIND, 8, 4>(a, s) : launch<KIND, 16, 2>(a, s);
    if (pieces <= 4096) return launch<KIND, 16, 4>(a, s);
    return launch<KIND, 16, 8>(a, s);
}

}  // namespace

hipError_t launch_rows(RowsKind kind, const RowsArgs& all, hipStream_t s)
{
    // A grid counts its threads in 32 bits: 2^21 rows of 1024 at a time.
    constexpr int kMost = 1 << 21;
    RowsArgs a = all;
    if (all.rows > kMost) {
        const auto moved = [](Rows r, int64_t rows, int bytes) { return r.p ? Rows{static_cast<char*>(r.p) + rows * r.stride * bytes, r.stride} : r; };
        const int wide = kind == kNormSum32 ? 4 : 2;
        for (int64_t at = 0; at < all.rows; at += kMost) {
            a.a = moved(all.a, at, 2);
            a.b = moved(all.b, at, wide);
            a.sum = moved(all.sum, at, wide);
            a.y = moved(all.y, at, 2);
            if (a.out.codes) a.out = {all.out.codes + at * all.out.stride, all.out.scales + at, all.out.stride};
            a.rows = all.rows - at < kMost ? int(all.rows - at) : kMost;
            if (const hipError_t e = launch_rows(kind, a, s); e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    switch (kind) {
    case kPlainRows: return launch_kind<kPlainRows>(a, s);
    case kGatedRows: return launch_kind<kGatedRows>(a, s);
    case kNormRows: return launch_kind<kNormRows>(a, s);
    case kNormSum16: return launch_kind<kNormSum16>(a, s);
    default: return launch_kind<kNormSum32>(a, s);
    }
}

}  // namespace tl
