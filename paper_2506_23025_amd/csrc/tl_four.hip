// Products with 4-bit weights and group scales.
#include "tl_rows.hpp"

#include <cmath>

namespace tl {
namespace {

constexpr int64_t kLimit = 0x7ffffff0;      // a descriptor's size: less than any offset that is none
constexpr int kRawBuffer = 0x00027000;      // a descriptor's last word: bytes, no format, no swizzle

// The eight weights of a packed word in order, less what `less` (the negated 1024 + z twice, and 64 + z twice) holds.  A code in the lowest four bits of fp16's 1024 is 1024 + code,
// one four bits further up in 64's mantissa 64 + code, and both differences are exact: no shift for half of the codes.
// The masks and bases are kept from the compiler, which would write each into two instructions instead of one for both.
struct Decode {
    uint32_t mask0 = 0x000F000Fu, mask4 = 0x00F000F0u, base1024 = 0x64006400u, base64 = 0x54005400u;
    __device__ Decode() { asm("" : "+s"(mask0), "+s"(mask4), "+v"(base1024), "+v"(base64)); }
    __device__ inline f16x8 operator()(uint32_t w, f16x2 less1024, f16x2 less64) const
    {
        const auto pair = [](uint32_t u, uint32_t mask, uint32_t base, f16x2 less) { return __builtin_bit_cast(f16x2, (u & mask) | base) + less; };
        const uint32_t v = w >> 8;
        const f16x2 a = pair(w, mask0, base1024, less1024), b = pair(w, mask4, base64, less64);
        const f16x2 c = pair(v, mask0, base1024, less1024), d = pair(v, mask4, base64, less64);
        return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
};

// Rows of less than eight places, which is what the other kernel fetches at a time: 16 columns of y and 16 rows, the groups dealt to four waves.
__global__ void __launch_bounds__(256) simple_kernel(Gemm4Desc g)
{
    __shared__ f32x4 part[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t n0 = int64_t(blockIdx.x) * 16 + (lane & 15), n = n0 < g.N ? n0 : g.N - 1;
    const int64_t m0 = int64_t(blockIdx.y) * 16 + (lane & 15), m = m0 < g.M ? m0 : g.M - 1;
    const uint32_t* const w = g.W + n * ((g.K + 127) / 128 * 16);
    const _Float16* const x = g.x + m * g.K;
    const int64_t groups = (g.K + g.group - 1) / g.group;
    const Decode decoded;
    f32x4 total = {0, 0, 0, 0};
    for (int64_t j = wave; j < groups; j += 4) {
        const int z = g.zeros ? g.zeros[j * g.N + n] : 8;
        const _Float16 less1024 = _Float16(-1024 - z), less64 = _Float16(-64 - z);
        f32x4 sum = {0, 0, 0, 0};
        const int64_t end = (j + 1) * g.group < g.K ? (j + 1) * g.group : g.K;
        for (int64_t k = j * g.group; k < end; k += 32) {
            const int64_t word = (k >> 5 & 3) + (lane >> 4) * 4;          // place of word 4 (k / 32 % 4) + lane / 16 of its block
            f16x8 a = {};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t at = k + (lane >> 4) * 8 + i;
                a[i] = at < end ? x[at] : _Float16(0.0f);
            }
            const f16x8 b = decoded(w[k / 128 * 16 + word], f16x2{less1024, less1024}, f16x2{less64, less64});
            sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, sum, 0, 0, 0);
        }
        const float scale = float(g.scales[j * g.N + n]);
        total += sum * scale;
    }
    part[wave][lane] = total;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 1; i < 4; ++i) total += part[i][lane];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = int64_t(blockIdx.y) * 16 + (lane >> 4) * 4 + i;
        if (row >= g.M || n0 >= g.N) continue;
        if (g.wide) static_cast<float*>(g.y)[row * g.N + n] = total[i];
        else static_cast<_Float16*>(g.y)[row * g.N + n] = _Float16(total[i]);
    }
}

typedef u32x4 __attribute__((aligned(2))) u32x4_any;

// Eight fp16 less the first n of them, 0 behind: what a piece that was fetched n values early holds.
__device__ inline u32x4 shifted(u32x4 v, int n)
{
    if (n & 4) v = u32x4{v[2], v[3], 0, 0};
    if (n & 2) v = u32x4{v[1], v[2], v[3], 0};
    if (n & 1) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
    return n < 8 ? v : u32x4{0, 0, 0, 0};
}

// Up to MR rows and 16 FN WN columns of y a workgroup.  K goes by chunks of 128, dealt to WK sets of waves; a wave has FN column fragments, and their words come straight into its
// registers, D chunks ahead.  Rows of x go through registers into LDS, a panel of CP WK chunks at a time and the next one while a panel is used, since every wave needs all of them; a panel's scales
// and zeros go the same way, as a wave that fetched its own would ask for 32 bytes four times over at every turn.
// The words are the column operand of the matrix instruction: a lane has one column, so one zero point and one scale.  Sums of UNIT steps of 32 are scaled and added in fp32.
// What bounds it (MI355X, weights out of the caches): one row memory, 32000 x 4096 14.0 us = 5.7 TB/s without the launch's 2.5, 4096 x 4096 4.2; the decode before that (masks and bases as literals, 13
// instead of 9 instructions a word: 15.4 and 4.7).  More rows what every workgroup fetches of x: 24 rows of 32000 x 4096 21.7 us (16.6 to 17.5 where some of the 65 MB are in the caches), 64 rows of 4096 x 4096 9.0.  More chunks ahead, and all columns' sums
// in one wave, made no difference or less.
template <int MR, int FN, int WN, int WK, int CP, int D, int UNIT, bool ZEROS>
__global__ void __launch_bounds__(64 * WN * WK) four_kernel(Gemm4Desc g)
{
    constexpr int FM = (MR + 15) / 16, THREADS = 64 * WN * WK, PK = CP * WK, XL = (MR * PK * 16 + THREADS - 1) / THREADS, FOLDS = 4 / UNIT;
    constexpr int BN = 16 * FN * WN, ENTRIES = PK * FOLDS * BN, SL = (ENTRIES + THREADS - 1) / THREADS, PANEL = MR * PK * 256 + ENTRIES * 4;
    static_assert(MR < 16 || MR % 16 == 0, "rows");
    static_assert(CP % D == 0 || D == 1, "register slots are known to the compiler");
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), quarter = lane >> 4, in = lane & 15;
    const int set = wave / WN, wn = wave % WN;
    const int n0 = (int(blockIdx.x) * WN + wn) * (16 * FN), m0 = int(blockIdx.y) * MR;
    const int K = int(g.K), N = int(g.N);
    const int chunks = (K + 127) >> 7, panels = (chunks + PK - 1) / PK;
    const int rows = int(g.M) - m0 < MR ? int(g.M) - m0 : MR;
    const uint32_t blocks32 = uint32_t(K + 31) >> 5;

    // ---- words of a chunk ------------------------------------------------------------------------------------
    const int64_t row_bytes = int64_t(chunks) * 64, wleft = (int64_t(N) - n0) * row_bytes;
    const auto wbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint32_t*>(g.W) + n0 * (row_bytes / 4), 0, int(wleft < kLimit ? (wleft > 0 ? wleft : 0) : kLimit), kRawBuffer);
    uint32_t woff[FN];
#pragma unroll
    for (int f = 0; f < FN; ++f) {
        const int n = 16 * f + in, last = N - 1 - n0;
        woff[f] = uint32_t(n < last ? n : (last > 0 ? last : 0)) * uint32_t(row_bytes) + uint32_t(quarter) * 16u;
    }
    struct Slot { u32x4 w[FN]; } slots[D];
    const auto load = [&](Slot& b, int chunk) {
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t o = chunk < chunks ? uint32_t(chunk) * 64u : 0x80000000u;
#pragma unroll
        for (int f = 0; f < FN; ++f) b.w[f] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wbuf, int(woff[f] + o), 0, 0));
        __builtin_amdgcn_sched_barrier(0);
    };

    // ---- rows of a panel: piece i of a thread is eight places of a row ----------------------------------------------
    u32x4 xr[XL];
    uint16_t sr[SL];
    uint8_t zr[SL];
    const auto fetch = [&](int panel) {
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int at = i * THREADS + tid, r = at / (PK * 16), k = panel * (PK * 128) + (at % (PK * 16)) * 8;
            const int64_t row = int64_t(m0) + (r < rows ? r : rows - 1);
            xr[i] = *reinterpret_cast<const u32x4_any*>(g.x + row * K + (k < K - 8 ? k : K - 8));
        }
        // a column's scale and zero for every UNIT blocks of 32 places
#pragma unroll
        for (int i = 0; i < SL; ++i) {
            const int at = i * THREADS + tid, c = at % BN + int(blockIdx.x) * BN;
            const uint32_t block = uint32_t(panel * (PK * 4) + at / BN * UNIT), group = uint32_t(uint64_t(block < blocks32 ? block : blocks32 - 1) * g.magic >> 31);
            const int64_t from = int64_t(group) * N + (c < N ? c : N - 1);
            sr[i] = reinterpret_cast<const uint16_t*>(g.scales)[from];
            if constexpr (ZEROS) zr[i] = g.zeros[from];
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto place = [&](int panel) {
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int at = i * THREADS + tid, r = at / (PK * 16), p = at % (PK * 16), k = panel * (PK * 128) + p * 8;
            u32x4 v = xr[i];
            if (K % 8 != 0) v = shifted(v, k < K - 8 ? 0 : k - (K - 8) < 8 ? k - (K - 8) : 8);
            else v = k < K ? v : u32x4{0, 0, 0, 0};
            if (MR * PK * 16 % THREADS == 0 || r < MR)
                *reinterpret_cast<u32x4*>(lds + (panel & 1) * PANEL + r * (PK * 256) + (p >> 4) * 256 + ((p ^ r) & 15) * 16) = v;
        }
#pragma unroll
        for (int i = 0; i < SL; ++i) {
            const int at = i * THREADS + tid;
            uint32_t v = uint32_t(panel * (PK * 4) + at / BN * UNIT) < blocks32 ? sr[i] : 0u;      // nothing behind K: an infinite scale would make its 0 a NaN
            if constexpr (ZEROS) v |= uint32_t(__builtin_bit_cast(uint16_t, _Float16(short(zr[i])))) << 16;
            if (ENTRIES % THREADS == 0 || at < ENTRIES) reinterpret_cast<uint32_t*>(lds + (panel & 1) * PANEL + MR * PK * 256)[at] = v;
        }
    };
    uint32_t xread[4];                                    // of the four steps of a chunk; rows that there are not hold another's places
    const int xrow = MR < 16 && in >= MR ? MR - 1 : in;
#pragma unroll
    for (int t = 0; t < 4; ++t) xread[t] = uint32_t(xrow) * (PK * 256) + uint32_t((4 * t + quarter) ^ xrow) * 16u;

    const Decode decoded;
    f32x4 total[FM][FN];
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int f = 0; f < FN; ++f) total[a][f] = f32x4{0, 0, 0, 0};
    const auto use = [&](const Slot& b, int panel, int local) {
        const unsigned char* const xs = lds + (panel & 1) * PANEL;
        // all reads, all decodes, all products: the decodes take as long as the reads do
        f16x8 x[4][FM], w[4][FN];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int a = 0; a < FM; ++a) x[t][a] = *reinterpret_cast<const f16x8*>(xs + xread[t] + a * (16 * PK * 256) + local * 256);
        f16x2 sz[FN][FOLDS];                              // scale, zero
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int h = 0; h < FOLDS; ++h)
                sz[f][h] = *reinterpret_cast<const f16x2*>(xs + MR * PK * 256 + ((local * FOLDS + h) * BN + wn * (16 * FN) + f * 16 + in) * 4);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const _Float16 z = ZEROS ? sz[f][t / UNIT][1] : _Float16(8);
                w[t][f] = decoded(b.w[f][t], f16x2{_Float16(-1024), _Float16(-1024)} - f16x2{z, z}, f16x2{_Float16(-64), _Float16(-64)} - f16x2{z, z});
            }
        __builtin_amdgcn_sched_barrier(0);
        f32x4 sum[FM][FN];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int f = 0; f < FN; ++f)
#pragma unroll
                for (int a = 0; a < FM; ++a) {
                    sum[a][f] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[t][a], w[t][f], t % UNIT == 0 ? f32x4{0, 0, 0, 0} : sum[a][f], 0, 0, 0);
                    if (t % UNIT == UNIT - 1) total[a][f] += sum[a][f] * float(sz[f][t / UNIT][0]);
                }
    };

    fetch(0);
#pragma unroll
    for (int d = 0; d < D; ++d) load(slots[d], d * WK + set);
    place(0);
    __syncthreads();
    const auto panel = [&](int p) {
#pragma unroll
        for (int c = 0; c < CP; ++c) {
            const int chunk = (p * CP + c) * WK + set;
            if (chunk < chunks) use(slots[c % D], p, c * WK + set);
            load(slots[c % D], chunk + D * WK);
        }
    };
    for (int p = 0; p < panels - 1; ++p) {
        fetch(p + 1);
        panel(p);
        place(p + 1);
        __syncthreads();
    }
    panel(panels - 1);

    // ---- the sets' sums, in their order ------------------------------------------------------------------------------
    const auto put = [&](f32x4 v, int a, int f, int n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = a * 16 + quarter * 4 + i;
            const int64_t c = int64_t(n) + f * 16 + in;
            if (r >= rows || c >= N) continue;
            const int64_t at = (int64_t(m0) + r) * N + c;
            if (g.wide) static_cast<float*>(g.y)[at] = v[i];
            else static_cast<_Float16*>(g.y)[at] = _Float16(v[i]);
        }
    };
    if constexpr (WK == 1) {
#pragma unroll
        for (int a = 0; a < FM; ++a)
#pragma unroll
            for (int f = 0; f < FN; ++f) put(total[a][f], a, f, n0);
    } else {
        constexpr int TILES = WN * FM * FN;
        f32x4* const part = reinterpret_cast<f32x4*>(lds);
        __syncthreads();
#pragma unroll
        for (int a = 0; a < FM; ++a)
#pragma unroll
            for (int f = 0; f < FN; ++f) part[(set * TILES + (wn * FM + a) * FN + f) * 64 + lane] = total[a][f];
        __syncthreads();
        for (int t = wave; t < TILES; t += WN * WK) {
            f32x4 v = part[t * 64 + lane];
#pragma unroll
            for (int i = 1; i < WK; ++i) v += part[(i * TILES + t) * 64 + lane];
            put(v, t / FN % FM, t % FN, (int(blockIdx.x) * WN + t / (FN * FM)) * (16 * FN));
        }
    }
}

template <int MR, int FN, int WN, int WK, int CP, int D>
struct Four {
    static constexpr int BN = 16 * FN * WN, RED = WK > 1 ? WN * WK * ((MR + 15) / 16) * FN * 1024 : 0;
    template <int UNIT, bool ZEROS>
    static hipError_t launch(const Gemm4Desc& g, hipStream_t s)
    {
        constexpr int PANEL = MR * CP * WK * 256 + CP * WK * (4 / UNIT) * BN * 4, MOST = 2 * PANEL > RED ? 2 * PANEL : RED;
        static_assert(MOST <= 160 * 1024, "LDS");
        if constexpr (MOST > 64 * 1024) {
            static std::atomic<uint64_t> set{0};
            const int device = device_slot();
            if (device < 0 || !(set.load(std::memory_order_relaxed) >> device & 1)) {
                if (const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(four_kernel<MR, FN, WN, WK, CP, D, UNIT, ZEROS>), hipFuncAttributeMaxDynamicSharedMemorySize, MOST); e != hipSuccess) return e;
                if (device >= 0) set.fetch_or(uint64_t(1) << device, std::memory_order_relaxed);
            }
        }
        if (g.M == 0) return hipSuccess;
        const int panels = (g.K + 128 * CP * WK - 1) / (128 * CP * WK) > 1 ? 2 : 1;
        const int lds = panels * PANEL > RED ? panels * PANEL : RED;
        hipLaunchKernelGGL((four_kernel<MR, FN, WN, WK, CP, D, UNIT, ZEROS>), dim3(unsigned((g.N + BN - 1) / BN), unsigned((g.M + MR - 1) / MR)), dim3(64 * WN * WK), lds, s, g);
        return hipGetLastError();
    }
    static hipError_t launch(const Gemm4Desc& g, hipStream_t s)
    {
        if (g.group % 128 == 0) return g.zeros ? launch<4, true>(g, s) : launch<4, false>(g, s);
        if (g.group % 64 == 0) return g.zeros ? launch<2, true>(g, s) : launch<2, false>(g, s);
        return g.zeros ? launch<1, true>(g, s) : launch<1, false>(g, s);
    }
};

// The time of a way, in us: rows, columns and K of a step of one workgroup, workgroups that a CU takes side by side, and what was fitted to 2 to 300 rows
// (launch, a step, a round, a round's step, a step of the rounds as a fraction but one at least, a round as a fraction).  The rows are dealt to several workgroups where there are few columns: at
// 64 x 4096 x 4096 32 rows a workgroup take 9.3 us and 64 rows, which leave half of the CUs without one, 14.0; at 64 x 1024 x 11008 32 rows 16.0, 16 rows 10.9 and 64 rows 32.0.  Over 5192 calls of N = 64 .. 65536,
// K = 256 .. 14336 and groups of 32 to 256 the way taken is 2.0 % slower than the best of 31 on average; over 1105 more calls 3.2 %, 12 % in one of twenty.
// Beyond 300 rows and below K = 256 the times are extrapolated; more than 192 rows have the ways of 64 alone to choose from, and every 64 rows read and decode the weights again.
struct WayTime {
    int rows, columns, step, per_cu;
    float c[6];
};
constexpr int kManyWays = 19;
constexpr WayTime kWayTimes[kManyWays] = {
    {1, 16, 1024, 1, {2.132f, 0.153f, 0.000f, 0.214f, 0.014f, 0.369f}},
    {4, 16, 1024, 1, {2.655f, 0.054f, 0.000f, 0.365f, 0.056f, 0.409f}},
    {8, 16, 1024, 2, {2.710f, 0.285f, 0.084f, 0.242f, 0.086f, 0.627f}},
    {8, 32, 1024, 1, {2.066f, 0.000f, 0.351f, 0.807f, 0.033f, 0.857f}},
    {8, 64, 512, 1, {1.940f, 0.000f, 0.292f, 0.724f, 0.000f, 1.129f}},
    {16, 16, 1024, 1, {2.083f, 0.350f, 0.000f, 0.455f, 0.108f, 0.395f}},
    {16, 32, 512, 3, {2.011f, 0.367f, 0.000f, 0.207f, 0.153f, 0.405f}},
    {16, 64, 512, 1, {2.068f, 0.000f, 0.199f, 0.804f, 0.033f, 1.021f}},
    {16, 128, 128, 1, {2.415f, 0.077f, 0.129f, 0.323f, 0.000f, 0.916f}},
    {32, 16, 1024, 1, {1.662f, 0.000f, 0.650f, 1.455f, 0.000f, 0.327f}},
    {32, 32, 512, 2, {2.093f, 0.360f, 0.094f, 0.377f, 0.233f, 0.368f}},
    {32, 64, 512, 1, {1.319f, 0.033f, 0.929f, 1.242f, 0.004f, 0.760f}},
    {32, 128, 256, 1, {1.174f, 0.000f, 1.208f, 0.924f, 0.002f, 1.586f}},
    {48, 32, 512, 1, {1.306f, 0.000f, 1.026f, 1.132f, 0.121f, 0.397f}},
    {48, 64, 512, 1, {1.278f, 0.025f, 1.493f, 1.627f, 0.000f, 0.666f}},
    {48, 128, 128, 1, {1.986f, 0.145f, 0.382f, 0.312f, 0.253f, 1.460f}},
    {64, 32, 512, 1, {1.573f, 0.003f, 0.878f, 1.615f, 0.000f, 0.408f}},
    {64, 64, 512, 1, {1.522f, 0.060f, 1.493f, 1.968f, 0.000f, 0.789f}},
    {64, 128, 128, 1, {1.512f, 0.090f, 1.148f, 0.771f, 0.000f, 1.590f}},
};
constexpr int kWays = kManyWays + 4;        // and those for one row alone

template <class F>
hipError_t with_way(int way, F&& f)
{
    switch (way) {
    case 0: return f(Four<1, 1, 1, 8, 4, 2>{});
    case 1: return f(Four<4, 1, 1, 8, 4, 4>{});
    case 2: return f(Four<8, 1, 1, 8, 4, 2>{});
    case 3: return f(Four<8, 1, 2, 8, 2, 2>{});
    case 4: return f(Four<8, 1, 4, 4, 2, 2>{});
    case 5: return f(Four<16, 1, 1, 8, 1, 1>{});
    case 6: return f(Four<16, 1, 2, 4, 1, 1>{});
    case 7: return f(Four<16, 1, 4, 4, 2, 2>{});
    case 8: return f(Four<16, 1, 8, 1, 8, 4>{});
    case 9: return f(Four<32, 1, 1, 8, 1, 1>{});
    case 10: return f(Four<32, 1, 2, 4, 1, 1>{});
    case 11: return f(Four<32, 2, 2, 4, 1, 1>{});
    case 12: return f(Four<32, 1, 8, 2, 2, 2>{});
    case 13: return f(Four<48, 1, 2, 4, 1, 1>{});
    case 14: return f(Four<48, 2, 2, 4, 1, 1>{});
    case 15: return f(Four<48, 1, 8, 1, 2, 2>{});
    case 16: return f(Four<64, 1, 2, 4, 1, 1>{});
    case 17: return f(Four<64, 2, 2, 4, 1, 1>{});
    case 18: return f(Four<64, 1, 8, 1, 2, 2>{});
    case 19: return f(Four<1, 1, 1, 8, 4, 4>{});
    case 20: return f(Four<1, 1, 1, 4, 8, 4>{});
    case 21: return f(Four<1, 1, 2, 4, 8, 2>{});
    default: return f(Four<1, 2, 2, 4, 8, 2>{});
    }
}

int way_of(int64_t M, int64_t N, int64_t K)
{
    if (M <= 1) {
        // by the column tiles of 16 that there are: few of them get all waves on their own part of K, many share the row's places among more columns (4096 x 4096 4.20 us with four sets of waves, 4.50
        // with eight; 4096 x 11008 7.8 and 7.1)
        const int64_t tiles = (N + 15) / 16;
        if (tiles <= 256 && K > 4096) return kManyWays;
        if (tiles < 256) return 0;
        return tiles < 768 ? kManyWays + 1 : tiles < 1536 ? kManyWays + 2 : kManyWays + 3;
    }
    int best = 0;
    float least = 0;
    for (int i = 0; i < kManyWays; ++i) {
        const WayTime& w = kWayTimes[i];
        if (w.rows < 64 && M > w.rows * 4) continue;
        const float r = float((M + w.rows - 1) / w.rows) * float((uint32_t(N) + uint32_t(w.columns) - 1) / uint32_t(w.columns)) * (1.0f / 256), k = float((uint32_t(K) + uint32_t(w.step) - 1) / uint32_t(w.step));
        const float turns = std::ceil(r > float(w.per_cu) ? r / float(w.per_cu) : r), rounds = r > float(w.per_cu) ? turns * float(w.per_cu) : turns;
        const float t = w.c[0] + w.c[1] * k + w.c[2] * rounds + w.c[3] * rounds * k + w.c[4] * (r > 1.0f ? r : 1.0f) * k + w.c[5] * r;
        if (least == 0 || t < least) least = t, best = i;
    }
    return best;
}

}  // namespace

hipError_t four_init()
{
    // one call of no rows for every way and form: it sets the kernel's limit for LDS
    for (int way = 0; way < kWays; ++way)
        for (const int64_t group : {32, 64, 128})
            for (int zeros = 0; zeros < 2; ++zeros) {
                Gemm4Desc g{nullptr, nullptr, nullptr, zeros ? reinterpret_cast<const uint8_t*>(&g) : nullptr, nullptr, 0, 16, 128, group, false, 0};
                if (const hipError_t e = with_way(way, [&](auto tile) { return decltype(tile)::launch(g, nullptr); }); e != hipSuccess) return e;
            }
    return hipSuccess;
}

int four_way(int64_t M, int64_t N, int64_t K) { return K < 8 ? -1 : way_of(M, N, K); }

hipError_t launch_gemm4(const Gemm4Desc& g, hipStream_t s)
{
    constexpr int64_t kRows = 65535;                      // what a grid's second dimension holds, of workgroups with one row each
    for (int64_t m = 0; m < g.M; m += kRows) {
        Gemm4Desc part = g;
        part.x += m * g.K;
        part.y = static_cast<char*>(g.y) + m * g.N * (g.wide ? 4 : 2);
        part.M = g.M - m < kRows ? g.M - m : kRows;
        part.magic = g.group >= g.K ? 0u : uint32_t(((uint64_t(1) << 31) + g.group / 32 - 1) / uint64_t(g.group / 32));
        if (g.K < 8) hipLaunchKernelGGL(simple_kernel, dim3(unsigned((g.N + 15) / 16), unsigned((part.M + 15) / 16)), dim3(256), 0, s, part);
        else if (const hipError_t e = with_way(way_of(part.M, g.N, g.K), [&](auto tile) { return decltype(tile)::launch(part, s); }); e != hipSuccess) return e;
    }
    return hipGetLastError();
}

}  // namespace tl
