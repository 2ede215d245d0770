// Ternary products over 8-bit rows: y = (codes . What^T) * (scale * gamma), the sum in whole numbers.
#include "tl_tile8.hpp"

#include <cmath>

namespace tl {
namespace {

// Tiles of 32 x 16 outputs of a launch of more than 16 rows: a grid counts its threads in 32 bits, and a workgroup of any way has 512 of them at most and one tile, also where that has fewer columns.
constexpr int64_t kMostTiles = int64_t(1) << 21;
constexpr int64_t kLimit = 0x7ffffff0;      // a descriptor's size: less than any offset that is none
constexpr int kRawBuffer = 0x00027000;      // a descriptor's last word: bytes, no format, no swizzle

// The value of the lane that DPP control CTRL names; 0 where there is none.
template <int CTRL>
__device__ inline int moved(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 15, 15, true); }

// Register j of quarter q of the wave (16 lanes) goes to register q of quarter j.
__device__ inline void transpose(u32x4& w)
{
    auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    w = u32x4{c[0], c[1], d[0], d[1]};
}


// What few rows need: 16 MB rows and 16 NB columns of y a workgroup, K in chunks of 256 dealt to NW waves, each of which has the whole tile, so that every code and every weight is
// read once a workgroup and straight into registers; D chunks are on their way.  The waves' sums meet in LDS.
// A matrix instruction's 16 rows of codes are as many different ones as there are, up to 16 / R, times R pieces of their places: one load brings the operands of R instructions, and each of these sums into
// registers of its own, of which it keeps the columns that its piece is in.
// What bounds it (MI355X, weights out of the caches): launch and memory's latency; 1 row of 2048 x 2048 2.6 us, of 14336 x 4096 5.5 (14.7 MB; without the pieces 6.3), of 4096 x 11008 5.0; at 16 rows the
// loads of x besides, 16 of 12288 x 4096 6.4 us.
template <int MB, int R, int NB, int NW, int D, int JOBS>
__global__ void __launch_bounds__(64 * NW) stream_kernel(Jobs8<JOBS> jobs)
{
    static_assert(R == 1 || MB == 1, "pieces beside each other");
    extern __shared__ __attribute__((aligned(16))) i32x4 part[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, in = lane & 15;
    const Job8& g = jobs.job[job_of(jobs)];
    int n0, m0;
    if constexpr (JOBS == 1) {
        n0 = int(blockIdx.x) * (16 * NB);
        m0 = int(blockIdx.y) * (16 * MB);
    } else {
        const int at = int(blockIdx.x) - g.first, down = g.down == 1 ? 0 : at / g.across;
        n0 = (at - down * g.across) * (16 * NB);
        m0 = down * (16 * MB);
    }
    const int words = (g.K + 15) >> 4, chunks = (words + 15) >> 4;
    // Loads through descriptors of what is left of W and x from the tile's first row on: addresses behind that give 0, and so does a chunk that is none.  Every load is
    // asked for without a branch, or the compiler, which has to know how many are on their way, waits for all of them.
    const int64_t wleft = (int64_t(g.N) - n0) * words * 4, xleft = (int64_t(g.M) - 1 - m0) * g.stride + words * 16;
    const auto wbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint32_t*>(g.W + size_t(n0) * words), 0, int(wleft < kLimit ? wleft : kLimit), kRawBuffer);
    const auto xbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(g.x + size_t(m0) * g.stride), 0, int(xleft < kLimit ? xleft : kLimit), kRawBuffer);
    uint32_t woff[NB], xoff[MB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int r = 16 * b + in, last = g.N - 1 - n0;
        woff[b] = uint32_t(r < last ? r : last) * uint32_t(words * 4) + uint32_t(quarter) * 16u;
    }
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        const int r = 16 * b + in % (16 / R), last = g.M - 1 - m0;
        xoff[b] = uint32_t(r < last ? r : last) * uint32_t(g.stride) + uint32_t(in / (16 / R)) * 64u + uint32_t(quarter) * 16u;
    }
    const int own = m0 + wave / NB * 16 + in;             // the row whose sums the wave closes with, where there are no more tiles than waves
    const float early = g.scales[own < g.M ? own : g.M - 1];
    constexpr int XL = 4 / R;                             // loads of a row block and chunk
    u32x4 w[D][NB];
    i32x4 x[D][MB][XL];
    const auto load = [&](int d, int chunk) {
        const uint32_t none = chunk < chunks ? 0u : 0x80000000u;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int b = 0; b < NB; ++b) w[d][b] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wbuf, int(woff[b] + (uint32_t(chunk) * 64u | none)), 0, 0));
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            const uint32_t o = xoff[b] + (uint32_t(chunk) * 256u | none);
#pragma unroll
            for (int j = 0; j < XL; ++j) x[d][b][j] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(xbuf, int(o + uint32_t(j) * (64u * R)), 0, 0));
        }
        __builtin_amdgcn_sched_barrier(0);                // in this order, or a wait for the first is one for all
    };
    i32x4 sum[R][MB][NB];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int a = 0; a < MB; ++a)
#pragma unroll
            for (int b = 0; b < NB; ++b) sum[r][a][b] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < D; ++d) load(d, wave + d * NW);
    for (int c = wave; c < chunks; c += D * NW) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int chunk = c + d * NW;
            if (chunk < chunks) {
                const int left = words - chunk * 16;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    if (left < 16) {                      // words behind the row's last stand for weights of 0
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[d][b][j] = quarter * 4 + j < left ? w[d][b][j] : 0x55555555u;
                    }
                    transpose(w[d][b]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        const i32x4 v = decoded8(w[d][b][j]);
#pragma unroll
                        for (int a = 0; a < MB; ++a) sum[j % R][a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v, x[d][a][j / R], sum[j % R][a][b], 0, 0, 0);
                    }
            }
            load(d, chunk + D * NW);
        }
    }
#pragma unroll
    for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            i32x4 s = sum[0][a][b];
#pragma unroll
            for (int i = 0; i < 4; ++i) {                 // from the lanes 16 / R, 2 * 16 / R, ... further on in the row of 16
                if constexpr (R == 2) s[i] += moved<0x108>(sum[1][a][b][i]);
                if constexpr (R == 4) s[i] += moved<0x104>(sum[1][a][b][i]) + moved<0x108>(sum[2][a][b][i]) + moved<0x10C>(sum[3][a][b][i]);
            }
            part[((a * NB + b) * NW + wave) * 64 + lane] = s;
        }
    __syncthreads();
    for (int t = wave; t < MB * NB; t += NW) {
        i32x4 s = part[t * NW * 64 + lane];
#pragma unroll
        for (int i = 1; i < NW; ++i) s += part[(t * NW + i) * 64 + lane];
        const int row = m0 + t / NB * 16 + in, col = n0 + t % NB * 16 + quarter * 4;
        if (row >= g.M || (R > 1 && in >= 16 / R)) continue;
        const float scale = (MB * NB <= NW ? early : g.scales[row]) * g.gamma;
        __half h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __float2half_rn(rounded(float(s[i]) * scale));
        __half* const y = g.y + size_t(row) * g.N + col;
        if (g.N % 4 == 0 && col < g.N) {
            *reinterpret_cast<u32x2*>(y) = *reinterpret_cast<const u32x2*>(h);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i < g.N) y[i] = h[i];
        }
    }
}

// ---- the ways of a launch: rows and columns of a workgroup's tile, places that it takes a step, workgroups a CU -----------------------------

template <int MB, int R, int NB, int NW, int D>
struct Stream {
    static constexpr int BM = 16 * MB, BN = 16 * NB, THREADS = 64 * NW;
    template <int JOBS>
    static hipError_t launch(const Jobs8<JOBS>& jobs, int64_t groups, hipStream_t s)
    {
        constexpr int lds = MB * NB * NW * 1024;
        static_assert(lds <= 64 * 1024, "no attribute to set");
        if (groups == 0) return hipSuccess;
        const Job8& g = jobs.job[0];
        hipLaunchKernelGGL((stream_kernel<MB, R, NB, NW, D, JOBS>), JOBS == 1 ? dim3(unsigned(g.across), unsigned(g.down)) : dim3(unsigned(groups)), dim3(64 * NW), lds, s, jobs);
        return hipGetLastError();
    }
};
template <int FM, int FN, int WM, int WN, int WK, int ST, bool RAGGED>
struct Tile {
    using C = Tile8Cfg<FM, FN, WM, WN, WK, ST, RAGGED>;
    static constexpr int BM = C::BM, BN = C::BN, THREADS = 64 * C::WAVES;
    template <int JOBS>
    static hipError_t launch(const Jobs8<JOBS>& jobs, int64_t groups, hipStream_t s) { return launch_tile8<C, JOBS>(jobs, groups, s); }
};

// Up to kMaxJobs products in one launch of a way.
template <class Way>
hipError_t launch_way(const Gemm8Desc* const* list, int count, hipStream_t s)
{
    Jobs8<kMaxJobs> all{};
    int64_t groups = 0;
    for (int i = 0; i < kMaxJobs; ++i) all.first[i] = 0x7fffffff;
    for (int i = 0; i < count; ++i) {
        const Gemm8Desc& g = *list[i];
        const int64_t across = (g.N + Way::BN - 1) / Way::BN, down = (g.M + Way::BM - 1) / Way::BM;
        all.job[i] = {g.x.codes, g.x.scales, g.W, g.y, g.gamma, int(g.M), int(g.N), int(g.K), int(g.x.stride), int(groups), int(across), int(down)};
        all.first[i] = int(groups);
        groups += across * down;
    }
    if (count == 1 && all.job[0].down < 65536)            // what a grid's second dimension holds
        return Way::template launch<1>({{0}, {all.job[0]}}, groups, s);
    return Way::template launch<kMaxJobs>(all, groups, s);
}

// Which way.  Up to 16 rows: by the tiles of 16 columns that there are and the chunks of 256 places, since few tiles need all waves of the chip on one and many do not.  Measured over calls
// of 1 to 3 products, N = 64 .. 22016, K = 128 .. 14336: the way taken is 1.4 % slower than the best of 12 on average with up to 4 rows (1150 calls), 2 % and 1.6 % slower than the best of 10 with 5 to 8 (500) and
// 9 to 16 (960), 8 % in one of twenty.
int few_way(const Gemm8Desc* const* list, int count)
{
    int64_t tiles = 0, M = 0, K = 0;
    for (int i = 0; i < count; ++i) {
        tiles += (list[i]->N + 15) / 16;
        M = list[i]->M > M ? list[i]->M : M;
        K = list[i]->K > K ? list[i]->K : K;
    }
    const int64_t chunks = (K + 255) / 256;
    if (M <= 4) {
        if (tiles >= 768) return chunks > 8 && tiles < 1024 ? 3 : 2;
        return chunks > 16 && tiles < 512 ? 1 : 0;
    }
    // As few columns a workgroup as leave one to a CU, or two, three, ...: 12288 x 4096 at M = 16 with 32 / 48 / 64 columns (384, 256, 192 workgroups) 8.7 / 6.4 / 7.0 us.
    const auto groups = [&](int nb) {
        int64_t n = 0;
        for (int i = 0; i < count; ++i) n += (list[i]->N + 16 * nb - 1) / (16 * nb);
        return n;
    };
    if (M <= 8) {
        if (tiles < 896) return chunks > 4 && tiles < 384 ? 5 : 4;
        const int64_t most = (groups(4) + 255) / 256 * 256;
        if (tiles < 1536 || groups(2) <= most) return 6;
        return groups(3) <= most ? 7 : 8;
    }
    const int64_t most = (groups(6) + 255) / 256 * 256;
    const int two = chunks > 8;
    for (int nb = 1; nb <= 4; ++nb)
        if (groups(nb) <= most) return 7 + 2 * nb + two;
    return chunks > 16 ? 18 : 17;
}
template <class F>
hipError_t with_few(int way, F&& f)
{
    switch (way) {
    case 0: return f(Stream<1, 4, 1, 8, 1>{});
    case 1: return f(Stream<1, 4, 1, 8, 2>{});
    case 2: return f(Stream<1, 4, 2, 4, 1>{});
    case 3: return f(Stream<1, 4, 2, 4, 2>{});
    case 4: return f(Stream<1, 2, 1, 4, 1>{});
    case 5: return f(Stream<1, 2, 1, 4, 2>{});
    case 6: return f(Stream<1, 2, 2, 4, 1>{});
    case 7: return f(Stream<1, 2, 3, 4, 1>{});
    case 8: return f(Stream<1, 2, 4, 4, 1>{});
    case 9: return f(Stream<1, 1, 1, 4, 1>{});
    case 10: return f(Stream<1, 1, 1, 4, 2>{});
    case 11: return f(Stream<1, 1, 2, 4, 1>{});
    case 12: return f(Stream<1, 1, 2, 4, 2>{});
    case 13: return f(Stream<1, 1, 3, 4, 1>{});
    case 14: return f(Stream<1, 1, 3, 4, 2>{});
    case 15: return f(Stream<1, 1, 4, 4, 1>{});
    case 16: return f(Stream<1, 1, 4, 4, 2>{});
    case 17: return f(Stream<1, 1, 6, 4, 1>{});
    default: return f(Stream<1, 1, 6, 4, 2>{});
    }
}

// More rows: what each way takes (us), fitted to 830 calls of M = 17 .. 4096, N and K as above, weights out of the caches: a launch and its steps, and a share for every round that the workgroups make of the chip
// (c: launch, a step, a round, a round's step, a step of the rounds as a fraction but one at least, a round as a fraction).  The way taken is 1.4 % slower than the best of 15 on average, 8 % in one of twenty.
struct WayTime {
    int bm, bn, ks, per_cu;
    double c[6];
};
constexpr int kWays = 11;
constexpr WayTime kWayTimes[kWays] = {
    {32, 16, 1024, 3, {1.763, 0.124, 0.000, 0.416, 0.240, 0.000}},
    {32, 32, 1024, 3, {1.964, 0.111, 0.000, 0.521, 0.239, 0.000}},
    {32, 32, 1024, 1, {1.359, 0.000, 1.666, 0.559, 0.000, 0.540}},
    {32, 64, 512, 1, {1.421, 0.000, 1.405, 0.442, 0.000, 0.717}},
    {64, 64, 512, 1, {1.392, 0.000, 2.307, 0.559, 0.000, 0.978}},
    {32, 128, 256, 2, {2.568, 0.162, 0.452, 0.235, 0.047, 0.989}},
    {64, 128, 512, 1, {1.846, 0.000, 2.461, 1.014, 0.000, 2.065}},
    {64, 128, 256, 2, {3.305, 0.170, 0.355, 0.274, 0.186, 1.774}},
    {128, 128, 256, 1, {1.005, 0.000, 4.436, 0.844, 0.000, 2.940}},
    {128, 128, 128, 2, {3.820, 0.099, 0.295, 0.216, 0.222, 1.769}},
    {128, 256, 128, 2, {3.469, 0.226, 0.000, 0.231, 0.493, 3.296}},
};

double way_time(int way, const Gemm8Desc* const* list, int count)
{
    const WayTime& w = kWayTimes[way];
    double groups = 0, steps = 0;
    for (int i = 0; i < count; ++i) {
        groups += double((list[i]->M + w.bm - 1) / w.bm) * double((list[i]->N + w.bn - 1) / w.bn);
        const double k = double((list[i]->K + w.ks - 1) / w.ks);
        steps = k > steps ? k : steps;
    }
    const double r = groups / 256.0, rounds = r > w.per_cu ? std::ceil(r / w.per_cu) * w.per_cu : std::ceil(r);
    return w.c[0] + w.c[1] * steps + w.c[2] * rounds + w.c[3] * rounds * steps + w.c[4] * (r > 1.0 ? r : 1.0) * steps + w.c[5] * r;
}

int best_way(const Gemm8Desc* const* list, int count, double* time)
{
    int best = 0;
    for (int i = 0; i < kWays; ++i) {
        const double t = way_time(i, list, count);
        if (i == 0 || t < *time) *time = t, best = i;
    }
    return best;
}

template <bool RAGGED, class F>
hipError_t with_tile(int way, F&& f)
{
    switch (way) {
    case 2: return f(Tile<2, 2, 1, 1, 8, 4, RAGGED>{});
    case 3: return f(Tile<2, 2, 1, 2, 4, 4, RAGGED>{});
    case 4: return f(Tile<4, 2, 1, 2, 4, 4, RAGGED>{});
    case 5: return f(Tile<2, 2, 1, 4, 2, 4, RAGGED>{});
    case 6: return f(Tile<4, 4, 1, 2, 4, 3, RAGGED>{});
    case 7: return f(Tile<4, 2, 1, 4, 2, 3, RAGGED>{});
    case 8: return f(Tile<4, 4, 2, 2, 2, 4, RAGGED>{});
    case 9: return f(Tile<4, 4, 2, 2, 1, 4, RAGGED>{});
    default: return f(Tile<8, 4, 1, 4, 1, 3, RAGGED>{});
    }
}
template <class F>
hipError_t with_many(int way, bool ragged, F&& f)
{
    if (way == 0) return f(Stream<2, 1, 1, 4, 1>{});
    if (way == 1) return f(Stream<2, 1, 2, 4, 1>{});
    return ragged ? with_tile<true>(way, f) : with_tile<false>(way, f);
}

// The launch that products share.
struct Launch8 {
    bool few, ragged;                     // up to 16 rows; packed rows that are no multiple of 16 bytes
    int way, count;
    const Gemm8Desc* const* list;
    template <class F>
    hipError_t with(F&& f) const { return few ? with_few(way, f) : with_many(way, ragged, f); }
};
int64_t tiles_of(const Gemm8Desc& g) { return (g.M + 31) / 32 * ((g.N + 15) / 16); }
Launch8 launch_few(const Gemm8Desc* const* list, int count) { return {true, false, few_way(list, count), count, list}; }
Launch8 launch_many(int way, const Gemm8Desc* const* list, int count)
{
    bool ragged = false;
    for (int i = 0; i < count; ++i) ragged |= (list[i]->K + 15) / 16 % 4 != 0;
    return {false, ragged, way, count, list};
}

// The launches of a call, one after the other.
template <class F>
hipError_t each_launch(const Gemm8Desc* jobs, int64_t count, F&& f)
{
    // Products of up to 16 rows share launches; those of more do where that is expected to be faster.
    const Gemm8Desc* few[kMaxJobs];
    const Gemm8Desc* many[kMaxJobs];
    int nfew = 0, nmany = 0;
    const auto close_few = [&] {
        const hipError_t e = nfew ? f(launch_few(few, nfew)) : hipSuccess;
        nfew = 0;
        return e;
    };
    const auto close_many = [&] {
        if (nmany == 0) return hipSuccess;
        double apart = 0.0, together = 0.0, t = 0.0;
        int64_t tiles = 0;
        int own[kMaxJobs];
        for (int i = 0; i < nmany; ++i) {
            own[i] = best_way(many + i, 1, &t);
            apart += t;
            tiles += tiles_of(*many[i]);
        }
        const int way = best_way(many, nmany, &together);
        const int n = nmany;
        nmany = 0;
        if (together <= apart && tiles <= kMostTiles) return f(launch_many(way, many, n));
        for (int i = 0; i < n; ++i)
            if (const hipError_t e = f(launch_many(own[i], many + i, 1)); e != hipSuccess) return e;
        return hipSuccess;
    };
    for (int64_t i = 0; i < count; ++i) {
        const Gemm8Desc& g = jobs[i];
        if (g.M > 16 && tiles_of(g) > kMostTiles) {       // in launches of its own; 256 rows of the widest matrix are 2^23 tiles, which have 2^31 threads, as no way gives wide matrices more than 256 a tile
            const int64_t most = kMostTiles / ((g.N + 15) / 16) * 32, rows = most > 256 ? most / 256 * 256 : 256;
            for (int64_t m = 0; m < g.M; m += rows) {
                const Gemm8Desc part{{g.x.codes + m * g.x.stride, g.x.scales + m, g.x.stride}, g.W, g.y + m * g.N, g.gamma, g.M - m < rows ? g.M - m : rows, g.N, g.K};
                const Gemm8Desc* const one = &part;
                double t;
                if (const hipError_t e = f(launch_many(best_way(&one, 1, &t), &one, 1)); e != hipSuccess) return e;
            }
        } else if (g.M <= 16) {
            few[nfew++] = &g;
            if (nfew == kMaxJobs)
                if (const hipError_t e = close_few(); e != hipSuccess) return e;
        } else {
            many[nmany++] = &g;
            if (nmany == kMaxJobs)
                if (const hipError_t e = close_many(); e != hipSuccess) return e;
        }
    }
    if (const hipError_t e = close_few(); e != hipSuccess) return e;
    return close_many();
}

}  // namespace

hipError_t rows8_init()
{
    const Gemm8Desc none{{nullptr, nullptr, 0}, nullptr, nullptr, 0.0f, 0, 0, 64};
    const Gemm8Desc* const list[2] = {&none, &none};
    for (int way = 2; way < kWays; ++way)
        for (int count = 1; count <= 2; ++count)
            for (int ragged = 0; ragged < 2; ++ragged)
                if (const hipError_t e = with_many(way, ragged, [&](auto w) { return launch_way<decltype(w)>(list, count, nullptr); }); e != hipSuccess) return e;
    return hipSuccess;
}

hipError_t launch_rows8_jobs(const Gemm8Desc* jobs, int64_t count, hipStream_t s)
{
    return each_launch(jobs, count, [s](const Launch8& l) { return l.with([&](auto w) { return launch_way<decltype(w)>(l.list, l.count, s); }); });
}

int rows8_launches(const Gemm8Desc* jobs, int count, int64_t* out, int most)
{
    int n = 0;
    const hipError_t none = each_launch(jobs, count, [&](const Launch8& l) {
        return l.with([&](auto w) {
            using Way = decltype(w);
            int64_t groups = 0, rows = 0;
            for (int i = 0; i < l.count; ++i) {
                groups += ((l.list[i]->M + Way::BM - 1) / Way::BM) * ((l.list[i]->N + Way::BN - 1) / Way::BN);
                rows += l.list[i]->M;
            }
            const int64_t now[7] = {l.few, l.way, l.ragged, l.count, rows, groups, Way::THREADS};
            for (int i = 0; n < most && i < 7; ++i) out[n * 7 + i] = now[i];
            ++n;
            return hipSuccess;
        });
    });
    return none == hipSuccess ? n : -1;
}

}  // namespace tl
