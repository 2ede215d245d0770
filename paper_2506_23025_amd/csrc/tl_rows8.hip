// Ternary products over 8-bit rows: y = (codes . What^T) * (scale * gamma), the sum in whole numbers.
#include "tl_rows.hpp"

namespace tl {
namespace {

// The 16 weights of a packed word, raised by 1, as four registers of four bytes: byte i of register s is weight 4 i + s, as the rows' codes stand.
__device__ inline i32x4 decoded(uint32_t w)
{
    return i32x4{int(w & 0x03030303u), int(w >> 2 & 0x03030303u), int(w >> 4 & 0x03030303u), int(w >> 6 & 0x03030303u)};
}

// 16 columns of y and 16 rows, the sum over K dealt to four waves.
__global__ void __launch_bounds__(256) simple_kernel(Gemm8Desc g)
{
    __shared__ i32x4 part[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t n = int64_t(blockIdx.x) * 16 + (lane & 15), m = int64_t(blockIdx.y) * 16 + (lane & 15);
    const int64_t words = (g.K + 15) / 16;
    const uint32_t* const w = g.W + (n < g.N ? n : g.N - 1) * words;
    const int8_t* const x = g.x.codes + (m < g.M ? m : g.M - 1) * g.x.stride;
    i32x4 sum = {0, 0, 0, 0};
    const i32x4 less = {-1, -1, -1, -1};                  // bytes of -1: takes the 1 away by which weights are raised
    for (int64_t k = int64_t(wave) * 4; k < words; k += 16) {
        const int64_t at = k + (lane >> 4);
        i32x4 b = {0, 0, 0, 0};
        uint32_t word = 0;
        if (at < words) {
            b = *reinterpret_cast<const i32x4*>(x + at * 16);
            word = w[at];
        }
        const i32x4 a = decoded(word);
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, sum, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(less, b, sum, 0, 0, 0);
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 1; i < 4; ++i) sum += part[i][lane];
    const int64_t row = int64_t(blockIdx.y) * 16 + (lane & 15);
    if (row >= g.M) return;
    const float scale = g.x.scales[row] * g.gamma;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t col = int64_t(blockIdx.x) * 16 + (lane >> 4) * 4 + i;
        if (col < g.N) g.y[row * g.N + col] = __float2half_rn(rounded(float(sum[i]) * scale));
    }
}

}  // namespace

hipError_t launch_rows8_jobs(const Gemm8Desc* jobs, int64_t count, hipStream_t s)
{
    for (int64_t i = 0; i < count; ++i) {
        const Gemm8Desc& g = jobs[i];
        constexpr int64_t kRows = int64_t(65535) * 16;
        for (int64_t m = 0; m < g.M; m += kRows) {
            Gemm8Desc part = g;
            part.x.codes += m * g.x.stride;
            part.x.scales += m;
            part.y += m * g.N;
            part.M = g.M - m < kRows ? g.M - m : kRows;
            hipLaunchKernelGGL(simple_kernel, dim3(unsigned((g.N + 15) / 16), unsigned((part.M + 15) / 16)), dim3(256), 0, s, part);
        }
    }
    return hipGetLastError();
}

}  // namespace tl
