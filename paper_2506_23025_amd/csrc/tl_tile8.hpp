// The tiled matrix-core kernel for many 8-bit rows: y = (codes . What^T) * (scale * gamma), the sum in whole numbers.
//
// A workgroup owns a BM x BN tile of y.  K is walked in blocks of 128 places; WK sets of WM x WN waves take a block each, a wave FM x FN fragments of
// v_mfma_i32_16x16x64_i8, two steps of 64 places to a block.  Rows and words go to LDS as they lie in memory, by LDS-DMA, ST blocks a set in the ring; a lane decodes the
// 16 weights of a word with 11 vector instructions between the products of the fragment before, and a decoded operand feeds FM of them.  The sums of the sets meet in LDS.
//
//  * What bounds it: at full size power and issue.  4096 x 14336 x 4096 (128 x 256 tiles, two workgroups a CU) 188 us = 2.56 POP/s at 1.96 GHz, the matrix pipes busy 62 %; a dense product in int8 of the
//    library's takes 232 us here.  Without the decode it is 3 % faster, without reads of x 5 %, without stores 4.5 %, without transfers 17 %.  256 x 256 tiles, one workgroup a CU: 196 us (nothing covers
//    a tile's end); 128 x 512 200.  In between, transfers from L2: 100 x 4096 x 11008 (32 x 64 tiles, 135 MB to LDS) 12.5 us.
//  * Transfers are spread between the products of a half (all of them right behind the barrier: 205 instead of 194 us with 256 x 256 tiles), without a branch: pieces behind the rows' end are fetched
//    from their beginning and met by weights of 0, so every step has as many transfers and one wait fits all.
//  * The barrier stands between the halves of a block, when the second half's operands are in registers or on their way.  No read of LDS is waited for at it.
//  * Words of a fragment's upper 8 columns stand with their two 16-byte pieces exchanged: 4-byte reads of 16 columns 32 bytes apart meet every bank once.
#pragma once
#include "tl_rows.hpp"
#include "tl_tile.hpp"

namespace tl {

// One product, and where its workgroups begin among a launch's.
struct Job8 {
    const int8_t* x;
    const float* scales;
    const uint32_t* W;
    __half* y;
    float gamma;
    int M, N, K;
    int stride;                           // bytes from row to row of x
    int first, across;                    // its first workgroup, and its workgroups along N
    int down;                             // along M
};
constexpr int kMaxJobs = 16;              // of a launch
template <int JOBS>
struct Jobs8 {
    int first[JOBS];                      // the jobs' first workgroups, or more than any: side by side, so that one load brings them
    Job8 job[JOBS];
};
// The job of this workgroup.
template <int JOBS>
__device__ inline int job_of(const Jobs8<JOBS>& jobs)
{
    int id = 0;
#pragma unroll
    for (int i = 1; i < JOBS; ++i) id += int(blockIdx.x) >= jobs.first[i];
    return id;
}

// The 16 weights of a packed word as four registers of four bytes: byte i of register s is weight 4 i + s, as the rows' codes stand.  A code picks its byte of a table.
__device__ inline i32x4 decoded8(uint32_t w)
{
    constexpr uint32_t table = 0x020100FFu, mask = 0x03030303u;
    return i32x4{int(__builtin_amdgcn_perm(0u, table, w & mask)), int(__builtin_amdgcn_perm(0u, table, w >> 2 & mask)),
                 int(__builtin_amdgcn_perm(0u, table, w >> 4 & mask)), int(__builtin_amdgcn_perm(0u, table, w >> 6 & mask))};
}

template <int FM_, int FN_, int WM_, int WN_, int WK_, int ST_, bool RAGGED_>
struct Tile8Cfg {
    static constexpr int FM = FM_, FN = FN_, WM = WM_, WN = WN_, WK = WK_, ST = ST_;
    static constexpr bool RAGGED = RAGGED_;                       // packed rows that are no multiple of 16 bytes
    static constexpr int WAVES = WM * WN * WK;
    static constexpr int BM = 16 * FM * WM, BN = 16 * FN * WN;
    static constexpr int XSET = BM * 128, WSET = BN * 32;         // a set's part of a stage
    static constexpr int STAGE = WK * (XSET + WSET);
    static constexpr int XD = XSET * WK / 1024 / WAVES;           // transfers of 1 KB a wave and stage
    static constexpr int WD = WSET * WK / (RAGGED ? 256 : 1024);  // transfers of 1 KB, or of 64 words, of all waves
    static constexpr int RED = WK > 1 ? WK * BM * BN * 4 : 0;
    static constexpr int PITCH = FN * 32 + 16;
    static constexpr int OUT = WK == 1 ? WAVES * 16 * PITCH : 0;
    static constexpr int LDS = STAGE * ST > RED ? (STAGE * ST > OUT ? STAGE * ST : OUT) : (RED > OUT ? RED : OUT);
    static constexpr int GROUPS = LDS <= 80 * 1024 && (FM * FN <= 8 || WAVES == 4) ? 2 : 1;   // workgroups a CU
    static_assert(XSET * WK % (1024 * WAVES) == 0 && WD % WAVES == 0, "every wave has as many transfers");
    static_assert(ST >= 3 && LDS <= 160 * 1024, "tile");
};

template <class C, int JOBS>
__global__ void __launch_bounds__(64 * C::WAVES) __attribute__((amdgpu_waves_per_eu(C::GROUPS * C::WAVES / 4, C::GROUPS * C::WAVES / 4)))
tile8_kernel(Jobs8<JOBS> jobs)
{
    using namespace tile;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    constexpr int FM = C::FM, FN = C::FN, BM = C::BM, BN = C::BN, WK = C::WK, ST = C::ST, WAVES = C::WAVES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, in = lane & 15;
    const int set = wave / (C::WM * C::WN), wm = wave / C::WN % C::WM, wn = wave % C::WN;
    const uint32_t lds0 = uint32_t(uintptr_t((const __attribute__((address_space(3))) unsigned char*)lds));

    const Job8& g = jobs.job[job_of(jobs)];

    // Workgroup ids go round the 8 XCDs, each with an L2 of its own: an XCD takes a contiguous piece of an order that walks the grid in bands of 4 row blocks, column by column.
    int tm, tn;
    {
        const int tiles_m = g.down, tiles_n = g.across, total = tiles_m * tiles_n, local = int(blockIdx.x) - g.first;
        const int xcd = local & 7, q = local >> 3, rem = total & 7;
        const int lin = xcd * (total >> 3) + (xcd < rem ? xcd : rem) + q;
        const int per_band = 4 * tiles_n, band = lin / per_band, r = lin - band * per_band;
        const int height = tiles_m - 4 * band < 4 ? tiles_m - 4 * band : 4;
        tn = r / height;
        tm = 4 * band + (r - tn * height);
    }
    const int m0 = tm * BM, n0 = tn * BN;
    const int words = (g.K + 15) >> 4, blocks = (words + 7) >> 3;        // blocks of 128 places: what a set takes a step
    const int steps = (blocks + WK - 1) / WK;

    // ---- transfers: 16-byte pieces of a row, 8 lanes to the 128 bytes of a block; pieces stand in LDS swizzled by row ------------
    const char* const xtile = reinterpret_cast<const char*>(g.x) + size_t(m0) * g.stride;
    const char* const wtile = reinterpret_cast<const char*>(g.W + size_t(n0) * words);
    const int mlast = g.M - 1 - m0, nlast = g.N - 1 - n0;
    const auto xrow = [&](int d) { return ((d * WAVES + wave) * 8 + (lane >> 3)) % BM; };
    const auto xset = [&](int d) { return ((d * WAVES + wave) * 8 + (lane >> 3)) / BM; };
    uint32_t xoff[C::XD];                                 // of the pieces of the first stage
#pragma unroll
    for (int d = 0; d < C::XD; ++d) {
        const int row = xrow(d);
        xoff[d] = uint32_t(row < mlast ? row : mlast) * uint32_t(g.stride) + uint32_t(xset(d) * 8 + piece_of<8>(row, lane & 7)) * 16u;
    }
    // Column c's two 16-byte pieces stand the other way round in the upper half of a fragment's 16 columns, so that a read of one piece of all of them meets every bank once.
    constexpr int WT = C::WD / WAVES;                     // a wave's transfers of weights
    const auto wword = [&](int d) {                       // the word that a transfer begins with, counted from its stage's first
        const int lin = (d * WAVES + wave) * 64 + lane, unit = C::RAGGED ? lin >> 2 : lin, col = unit / 2 % BN;
        return unit / 2 / BN * 8 + ((unit ^ col >> 3) & 1) * 4 + (C::RAGGED ? lin & 3 : 0);
    };
    uint32_t woff[WT];                                    // of the words of the first stage
#pragma unroll
    for (int d = 0; d < WT; ++d) {
        const int lin = (d * WAVES + wave) * 64 + lane, unit = C::RAGGED ? lin >> 2 : lin, col = unit / 2 % BN;
        woff[d] = (uint32_t(col < nlast ? col : nlast) * uint32_t(words) + uint32_t(wword(d))) * 4u;
    }
    // Stage s into a slot.  Pieces behind the row, of which stages behind the last have nothing else, are fetched from the row's beginning; their weights count as 0.
    constexpr int PER = C::XD + WT;                       // transfers of a wave and stage
    const auto issue = [&](int s, int slot, int first, int last) {
        const uint32_t to = lds0 + uint32_t(slot) * C::STAGE;
        // without a branch: as many transfers from every stage.  All of a wave's are of the same pieces where a stage is one set's
        const auto moved = [&](int from, int bytes) { return uint32_t(s * WK * 8 + from < words ? s * (WK * 8 * bytes) : -from * bytes); };
#pragma unroll
        for (int d = 0; d < C::XD; ++d) {
            if (d < first || d >= last) continue;
            const int e = WK == 1 ? 0 : d;
            dma16(xoff[d] + moved(xset(e) * 8 + piece_of<8>(xrow(e), lane & 7), 16), xtile, to + uint32_t(d * WAVES + wave) * 1024u);
        }
#pragma unroll
        for (int d = 0; d < WT; ++d) {
            const int i = d * WAVES + wave;
            if (C::XD + d < first || C::XD + d >= last) continue;
            const uint32_t at = to + WK * C::XSET + uint32_t(i) * (C::RAGGED ? 256u : 1024u), o = woff[d] + moved(wword(d), 4);
            if constexpr (C::RAGGED) dma4(o, wtile, at);
            else dma16(o, wtile, at);
        }
    };

    i32x4 sum[FM][FN];
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b) sum[a][b] = i32x4{0, 0, 0, 0};

    // Half a stage: 64 places, of which a lane has piece 4 j + quarter of its rows and that word of its columns.
    const unsigned char* const xread = lds + set * C::XSET + (wm * FM * 16 + in) * 128;
    const unsigned char* const wread = lds + WK * C::XSET + set * C::WSET + (wn * FN * 16 + in) * 32 + quarter * 4;
    const int flip = in >> 3 & 1;
    const uint32_t sw[2] = {uint32_t(slot_of<8>(in, quarter)) * 16u, uint32_t(slot_of<8>(in, 4 + quarter)) * 16u};
    struct Half { i32x4 x[FM]; uint32_t w[FN]; };
    const auto read_w = [&](Half& h, int slot, int j) {
#pragma unroll
        for (int b = 0; b < FN; ++b) h.w[b] = *reinterpret_cast<const uint32_t*>(wread + slot * C::STAGE + b * 512 + (j ^ flip) * 16);
    };
    const auto read_x = [&](Half& h, int slot, int j, int from, int to) {
#pragma unroll
        for (int a = from; a < to; ++a) h.x[a] = *reinterpret_cast<const i32x4*>(xread + slot * C::STAGE + a * 2048 + sw[j]);
    };
    const auto mask = [&](Half& h, int s, int j) {        // words behind the row's last stand for weights of 0
        const bool there = (s * WK + set) * 8 + 4 * j + quarter < words;
#pragma unroll
        for (int b = 0; b < FN; ++b) h.w[b] = there ? h.w[b] : 0x55555555u;
    };
    i32x4 v;                                              // the decoded operand in turn
    // The products of a half, a column fragment at a time; beside them the next half is read, its words first, and the next fragment decoded.
    const auto products = [&](const Half& h, Half& nh, int ns, int nslot, int nj, auto&& beside) {
#pragma unroll
        for (int b = 0; b < FN; ++b) {
            __builtin_amdgcn_sched_barrier(0);
            if (b == 0) read_w(nh, nslot, nj);
            read_x(nh, nslot, nj, b * FM / FN, (b + 1) * FM / FN);
            beside(b);
            if (b + 1 == FN) mask(nh, ns, nj);
            const i32x4 then = decoded8(b + 1 < FN ? h.w[b + 1] : nh.w[0]);
#pragma unroll
            for (int a = 0; a < FM; ++a) sum[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v, h.x[a], sum[a][b], 0, 0, 0);
            v = then;
        }
        __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) issue(s, s, 0, PER);
    wait_vm<(ST - 2) * PER>();
    asm volatile("s_barrier" : : : "memory");
    Half h0, h1;
    read_w(h0, 0, 0);
    read_x(h0, 0, 0, 0, FM);
    mask(h0, 0, 0);
    v = decoded8(h0.w[0]);
    int slot = 0;
    // Of a step: its first half; the next stage is there once every wave has seen its transfers end, and the stage before is free once every wave is past it; its second half.  The last
    // step reads on into a stage of nothing.
    for (int s = 0; s < steps; ++s) {
        const int next = slot + 1 < ST ? slot + 1 : 0, behind = slot ? slot - 1 : ST - 1;
        products(h0, h1, s, slot, 1, [](int) {});
        wait_vm<(ST - 3) * PER>();
        asm volatile("s_barrier" : : : "memory");
        products(h1, h0, s + 1, next, 0, [&](int b) { issue(s + ST - 1, behind, b * PER / FN, (b + 1) * PER / FN); });
        slot = next;
    }
    wait_vm<0>();

    if constexpr (WK > 1) {
        i32x4* const part = reinterpret_cast<i32x4*>(lds);
        lds_barrier();
        constexpr int TILES = C::WM * C::WN * FM * FN;
#pragma unroll
        for (int a = 0; a < FM; ++a)
#pragma unroll
            for (int b = 0; b < FN; ++b) part[(set * TILES + ((wm * C::WN + wn) * FM + a) * FN + b) * 64 + lane] = sum[a][b];
        lds_barrier();
        for (int t = wave; t < TILES; t += WAVES) {
            i32x4 v = part[t * 64 + lane];
#pragma unroll
            for (int i = 1; i < WK; ++i) v += part[(i * TILES + t) * 64 + lane];
            const int b = t % FN, a = t / FN % FM, cn = t / (FN * FM) % C::WN, cm = t / (FN * FM * C::WN);
            const int row = m0 + (cm * FM + a) * 16 + in, col = n0 + (cn * FN + b) * 16 + quarter * 4;
            if (row >= g.M) continue;
            const float scale = g.scales[row] * g.gamma;
            __half h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = __float2half_rn(rounded(float(v[i]) * scale));
            __half* const y = g.y + size_t(row) * g.N + col;
            if (g.N % 4 == 0 && col < g.N) {
                *reinterpret_cast<u32x2*>(y) = *reinterpret_cast<const u32x2*>(h);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (col + i < g.N) y[i] = h[i];
            }
        }
    } else {
        // 16 rows at a time through the wave's part of LDS, so that rows of y are written in 16-byte pieces
        lds_barrier();
        unsigned char* const turn = lds + wave * (16 * C::PITCH);
        constexpr int PIECES = FN * 2, ROUNDS = 16 * PIECES / 64;
        const int col0 = n0 + wn * FN * 16;
#pragma unroll
        for (int a = 0; a < FM; ++a) {
            const int base = m0 + (wm * FM + a) * 16;
            const int row = base + in;
            const float scale = g.scales[row < g.M ? row : g.M - 1] * g.gamma;
#pragma unroll
            for (int b = 0; b < FN; ++b) {
                f16x4 h;
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = _Float16(rounded(float(sum[a][b][i]) * scale));
                *reinterpret_cast<f16x4*>(turn + in * C::PITCH + b * 32 + quarter * 8) = h;
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r) {
                const int i = r * 64 + lane, tr = i / PIECES, piece = i % PIECES;
                const u32x4 v = *reinterpret_cast<const u32x4*>(turn + tr * C::PITCH + piece * 16);
                const int yr = base + tr, yc = col0 + piece * 8;
                if (yr >= g.M) continue;
                __half* const y = g.y + size_t(yr) * g.N + yc;
                if (g.N % 8 == 0 && yc < g.N) {
                    *reinterpret_cast<u32x4*>(y) = v;
                } else {
                    const f16x8 h = __builtin_bit_cast(f16x8, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (yc + e < g.N) y[e] = __half(h[e]);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
}

template <class C, int JOBS>
hipError_t launch_tile8(const Jobs8<JOBS>& jobs, int64_t groups, hipStream_t s)
{
    if constexpr (C::LDS > 64 * 1024) {
        static std::atomic<uint64_t> set{0};
        const int device = device_slot();
        if (device < 0 || !(set.load(std::memory_order_relaxed) >> device & 1)) {
            if (const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(tile8_kernel<C, JOBS>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS); e != hipSuccess) return e;
            if (device >= 0) set.fetch_or(uint64_t(1) << device, std::memory_order_relaxed);
        }
    }
    if (groups > 0) hipLaunchKernelGGL((tile8_kernel<C, JOBS>), dim3(unsigned(groups)), dim3(64 * C::WAVES), C::LDS, s, jobs);
    return hipGetLastError();
}

}  // namespace tl
