// Products with 4-bit weights and group scales.
#include "tl_rows.hpp"

namespace tl {
namespace {

// The eight weights of a packed word in order, less what `less` (the negated 1024 + z twice, and 64 + z twice) holds.  A code in the lowest four bits of fp16's 1024 is 1024 + code,
// one four bits further up in 64's mantissa 64 + code, and both differences are exact: no shift for half of the codes.
__device__ inline f16x8 decoded(uint32_t w, f16x2 less1024, f16x2 less64)
{
    const auto pair = [](uint32_t u, uint32_t mask, uint32_t base, f16x2 less) { return __builtin_bit_cast(f16x2, (u & mask) | base) + less; };
    const uint32_t v = w >> 8;
    const f16x2 a = pair(w, 0x000F000Fu, 0x64006400u, less1024), b = pair(w, 0x00F000F0u, 0x54005400u, less64);
    const f16x2 c = pair(v, 0x000F000Fu, 0x64006400u, less1024), d = pair(v, 0x00F000F0u, 0x54005400u, less64);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 16 columns of y and 16 rows, the groups dealt to four waves.
__global__ void __launch_bounds__(256) simple_kernel(Gemm4Desc g)
{
    __shared__ f32x4 part[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t n0 = int64_t(blockIdx.x) * 16 + (lane & 15), n = n0 < g.N ? n0 : g.N - 1;
    const int64_t m0 = int64_t(blockIdx.y) * 16 + (lane & 15), m = m0 < g.M ? m0 : g.M - 1;
    const uint32_t* const w = g.W + n * ((g.K + 127) / 128 * 16);
    const _Float16* const x = g.x + m * g.K;
    const int64_t groups = (g.K + g.group - 1) / g.group;
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

}  // namespace

hipError_t launch_gemm4(const Gemm4Desc& g, hipStream_t s)
{
    constexpr int64_t kRows = int64_t(65535) * 16;
    for (int64_t m = 0; m < g.M; m += kRows) {
        Gemm4Desc part = g;
        part.x += m * g.K;
        part.y = static_cast<char*>(g.y) + m * g.N * (g.wide ? 4 : 2);
        part.M = g.M - m < kRows ? g.M - m : kRows;
        hipLaunchKernelGGL(simple_kernel, dim3(unsigned((g.N + 15) / 16), unsigned((part.M + 15) / 16)), dim3(256), 0, s, part);
    }
    return hipGetLastError();
}

}  // namespace tl
