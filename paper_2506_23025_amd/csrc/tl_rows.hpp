// What the kernels over 8-bit rows and over 4-bit weights take, and their launchers.
#pragma once
#include "tl_internal.hpp"

#include <atomic>

namespace tl {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// A product or sum as fp32 rounds it, before it is rounded to fp16: the compiler joins the two into one instruction that rounds once.
__device__ inline float rounded(float x)
{
    asm("" : "+v"(x));
    return x;
}

struct Rows {
    void* p;
    int64_t stride;                       // in elements
};

struct Rows8 {
    int8_t* codes;
    float* scales;
    int64_t stride;                       // in bytes
};

struct RowsArgs {
    Rows a, b, sum, y;                    // norm: x, residual; gate: up, gate
    Rows8 out;
    const _Float16* weight;
    int rows, dim;
    double eps;
};

enum RowsKind { kPlainRows, kGatedRows, kNormRows, kNormSum16, kNormSum32 };
hipError_t launch_rows(RowsKind kind, const RowsArgs& a, hipStream_t s);

// One product over 8-bit rows, gamma already widened.
struct Gemm8Desc {
    Rows8 x;
    const uint32_t* W;
    __half* y;
    float gamma;
    int64_t M, N, K;
};
hipError_t launch_rows8_jobs(const Gemm8Desc* jobs, int64_t count, hipStream_t s);
hipError_t rows8_init();
// For the tests: the launches that launch_rows8_jobs makes, and of the first `most` of them: up to 16 rows or more (1, 0), way, odd packed rows, products, rows, workgroups, threads of one.
int rows8_launches(const Gemm8Desc* jobs, int count, int64_t* out, int most);

struct Gemm4Desc {
    const _Float16* x;
    const uint32_t* W;
    const _Float16* scales;
    const uint8_t* zeros;                 // NULL: 8
    void* y;
    int64_t M, N, K, group;
    bool wide;                            // y is fp32
    uint32_t magic;                       // 2^31 / (group / 32), rounded up, or 0 for one group: block * magic / 2^31 is the group of a block of 32 (blocks and groups are fewer than 2^15)
};
hipError_t launch_gemm4(const Gemm4Desc& g, hipStream_t s);            // sets magic itself
hipError_t four_init();
int four_way(int64_t M, int64_t N, int64_t K);                         // for the tests: the way of a product, or -1 for the kernel for K < 8

}  // namespace tl
