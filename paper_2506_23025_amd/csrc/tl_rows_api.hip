// C-ABI entry points of 8-bit rows and 4-bit weights: argument checks and launches; the 4-bit packer and quantiser on the host.
#include "tl_rows.hpp"

#include <cmath>

namespace tl {
namespace {

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
constexpr int64_t kMaxStride = int64_t(1) << 40, kMaxDim = 65536;
constexpr int64_t kMaxStride8 = int64_t(1) << 24;      // 256 rows lie within 32-bit offsets

// Rows of `bytes` a place that a call reads, or with `written` writes.
inline tl_status rows_status(const tl_rows& r, int64_t rows, int64_t dim, int bytes, bool written)
{
    if (!r.ptr) return TL_ERR_NULL;
    if (r.stride < 0 || r.stride >= kMaxStride || (written && rows > 1 && r.stride < dim)) return TL_ERR_SHAPE;
    if (!aligned(r.ptr, 16) || r.stride * bytes % 16 != 0) return TL_ERR_ALIGN;
    return TL_OK;
}

inline tl_status rows8_status(const tl_rows8& r, int64_t rows, int64_t dim)
{
    if (!r.codes || !r.scales) return TL_ERR_NULL;
    if (r.stride < 0 || r.stride >= kMaxStride8 || (rows > 1 && r.stride < (dim + 15) / 16 * 16)) return TL_ERR_SHAPE;
    if (!aligned(r.codes, 16) || r.stride % 16 != 0 || !aligned(r.scales, 4)) return TL_ERR_ALIGN;
    return TL_OK;
}

inline Rows rows_of(const tl_rows& r) { return {r.ptr, r.stride}; }
inline Rows8 rows8_of(const tl_rows8& r) { return {r.codes, r.scales, r.stride}; }

inline tl_status sizes_status(int64_t rows, int64_t dim)
{
    return rows < 0 || rows >= (int64_t(1) << 31) || dim < 1 || dim > kMaxDim ? TL_ERR_SHAPE : TL_OK;
}

inline bool product_ok(int64_t M, int64_t N, int64_t K)
{
    const int64_t lim = int64_t(1) << 31;
    return M >= 1 && N >= 1 && K >= 1 && M < lim && N < lim && K < lim && M * N < (int64_t(1) << 40) && N * K < (int64_t(1) << 42) && M * K < (int64_t(1) << 40);
}

inline tl_status from_hip(hipError_t e) { return e == hipSuccess ? TL_OK : TL_ERR_HIP; }

tl_status desc_of(const tl_gemm_rows8_job& j, Gemm8Desc& d)
{
    if (!j.Wpacked || !j.y) return TL_ERR_NULL;
    if (!product_ok(j.M, j.N, j.K) || j.N >= (int64_t(1) << 24) || j.K >= (int64_t(1) << 24)) return TL_ERR_SHAPE;
    if (const tl_status e = rows8_status(j.x, j.M, j.K); e != TL_OK) return e;
    if (!aligned(j.Wpacked, 16) || !aligned(j.y, 16)) return TL_ERR_ALIGN;
    d = {rows8_of(j.x), static_cast<const uint32_t*>(j.Wpacked), static_cast<__half*>(j.y), half_bits_to_float(j.gamma_fp16_bits), j.M, j.N, j.K};
    return TL_OK;
}

// ---- 4 bits on the host ----------------------------------------------------------------------

// To fp16, to the nearest, ties to even; false where the value is beyond it.
bool to_half(double v, uint16_t* bits, double* back)
{
    const _Float16 h = static_cast<_Float16>(v);
    *bits = __builtin_bit_cast(uint16_t, h);
    *back = static_cast<double>(static_cast<float>(h));
    return std::isfinite(*back);
}

inline bool group_ok(int64_t group) { return group >= 32 && group % 32 == 0 && group < (int64_t(1) << 31); }

inline int place_of(int word) { return 4 * (word % 4) + word / 4; }
inline int shift_of(int j) { return 4 * (j / 2) + 16 * (j % 2); }

}  // namespace
}  // namespace tl

extern "C" {

tl_status tl_norm(const tl_norm_job* job, void* stream)
{
    using namespace tl;
    if (!job) return TL_ERR_NULL;
    const tl_norm_job& j = *job;
    tl_status e = sizes_status(j.rows, j.dim);
    if (e != TL_OK) return e;
    if (code_of(j.real) != TL_REAL_FP16 && code_of(j.real) != TL_REAL_FP32) return TL_ERR_UNSUPPORTED;
    if (!(j.eps >= 0.0f) || !std::isfinite(j.eps)) return TL_ERR_VALUE;
    const int wide = j.real == TL_REAL_FP32 ? 4 : 2;
    const bool sum = j.residual.ptr && j.sum.ptr;
    if (!sum && !j.y.ptr && !j.out.codes) return TL_ERR_NULL;
    if ((e = rows_status(j.x, j.rows, j.dim, 2, false)) != TL_OK) return e;
    if (j.residual.ptr && (e = rows_status(j.residual, j.rows, j.dim, wide, false)) != TL_OK) return e;
    if (sum && (e = rows_status(j.sum, j.rows, j.dim, wide, true)) != TL_OK) return e;
    if (j.y.ptr && (e = rows_status(j.y, j.rows, j.dim, 2, true)) != TL_OK) return e;
    if (j.out.codes && (e = rows8_status(j.out, j.rows, j.dim)) != TL_OK) return e;
    if (!aligned(j.weight, 16)) return TL_ERR_ALIGN;
    if (j.rows == 0) return TL_OK;
    const RowsArgs a{rows_of(j.x), rows_of(j.residual), sum ? rows_of(j.sum) : Rows{nullptr, 0}, rows_of(j.y), rows8_of(j.out),
                     static_cast<const _Float16*>(j.weight), int(j.rows), int(j.dim), double(j.eps)};
    return from_hip(launch_rows(!j.residual.ptr ? kNormRows : wide == 4 ? kNormSum32 : kNormSum16, a, static_cast<hipStream_t>(stream)));
}

tl_status tl_gate(const tl_gate_job* job, void* stream)
{
    using namespace tl;
    if (!job) return TL_ERR_NULL;
    const tl_gate_job& j = *job;
    tl_status e = sizes_status(j.rows, j.dim);
    if (e != TL_OK) return e;
    if (!j.y.ptr && !j.out.codes) return TL_ERR_NULL;
    if ((e = rows_status(j.up, j.rows, j.dim, 2, false)) != TL_OK) return e;
    if (j.gate.ptr && (e = rows_status(j.gate, j.rows, j.dim, 2, false)) != TL_OK) return e;
    if (j.y.ptr && (e = rows_status(j.y, j.rows, j.dim, 2, true)) != TL_OK) return e;
    if (j.out.codes && (e = rows8_status(j.out, j.rows, j.dim)) != TL_OK) return e;
    if (j.rows == 0) return TL_OK;
    const RowsArgs a{rows_of(j.up), rows_of(j.gate), {nullptr, 0}, rows_of(j.y), rows8_of(j.out), nullptr, int(j.rows), int(j.dim), 0.0};
    return from_hip(launch_rows(j.gate.ptr ? kGatedRows : kPlainRows, a, static_cast<hipStream_t>(stream)));
}

tl_status tl_ternary_gemm_rows8(const tl_gemm_rows8_job* job, void* stream) { return job ? tl_ternary_gemm_rows8_grouped(job, 1, stream) : TL_ERR_NULL; }

tl_status tl_ternary_gemm_rows8_grouped(const tl_gemm_rows8_job* jobs, int64_t count, void* stream)
{
    using namespace tl;
    if (count < 0) return TL_ERR_SHAPE;
    if (count == 0) return TL_OK;
    if (!jobs) return TL_ERR_NULL;
    for (int64_t i = 0; i < count; ++i) {
        Gemm8Desc d;
        if (const tl_status e = desc_of(jobs[i], d); e != TL_OK) return e;
    }
    constexpr int kBatch = 64;            // nothing is allocated: so many at a time
    Gemm8Desc d[kBatch];
    for (int64_t at = 0; at < count; at += kBatch) {
        const int n = int(count - at < kBatch ? count - at : kBatch);
        for (int i = 0; i < n; ++i) desc_of(jobs[at + i], d[i]);
        if (const hipError_t e = launch_rows8_jobs(d, n, static_cast<hipStream_t>(stream)); e != hipSuccess) return TL_ERR_HIP;
    }
    return TL_OK;
}

size_t tl_row_stride_4bit(int64_t K) { return K < 1 || K >= (int64_t(1) << 40) ? 0 : size_t((K + 127) / 128) * 64; }

tl_status tl_quantize_4bit(const float* W, int64_t N, int64_t K, int64_t group, uint8_t* codes, uint16_t* scales, uint8_t* zeros)
{
    using namespace tl;
    if (!W || !codes || !scales) return TL_ERR_NULL;
    if (!product_ok(1, N, K) || !group_ok(group)) return TL_ERR_SHAPE;
    for (int64_t n = 0; n < N; ++n) {
        for (int64_t g = 0; g * group < K; ++g) {
            const float* const w = W + n * K + g * group;
            uint8_t* const c = codes + n * K + g * group;
            const int64_t count = K - g * group < group ? K - g * group : group;
            double lo = 0.0, hi = 0.0;
            for (int64_t i = 0; i < count; ++i) {
                if (!std::isfinite(w[i])) return TL_ERR_VALUE;
                lo = w[i] < lo ? w[i] : lo;
                hi = w[i] > hi ? w[i] : hi;
            }
            double s;
            if (!to_half(zeros ? (hi - lo) / 15.0 : (hi > -lo ? hi : -lo) / 7.0, &scales[g * N + n], &s)) return TL_ERR_VALUE;
            const auto held = [](double v) { return v < 0.0 ? 0.0 : v > 15.0 ? 15.0 : v; };
            const double z = zeros && s > 0.0 ? held(std::nearbyint(-lo / s)) : 8.0;
            if (zeros) zeros[g * N + n] = uint8_t(z);
            for (int64_t i = 0; i < count; ++i) c[i] = s > 0.0 ? uint8_t(held(z + std::nearbyint(w[i] / s))) : uint8_t(8);
        }
    }
    return TL_OK;
}

tl_status tl_pack_4bit(const uint8_t* codes, int64_t N, int64_t K, uint32_t* out)
{
    using namespace tl;
    if (!codes || !out) return TL_ERR_NULL;
    if (!product_ok(1, N, K)) return TL_ERR_SHAPE;
    const int64_t blocks = (K + 127) / 128;
    for (int64_t n = 0; n < N; ++n) {
        for (int64_t b = 0; b < blocks; ++b) {
            for (int w = 0; w < 16; ++w) {
                uint32_t word = 0;
                for (int j = 0; j < 8; ++j) {
                    const int64_t k = b * 128 + w * 8 + j;
                    const uint32_t c = k < K ? codes[n * K + k] : 0;
                    if (c > 15) return TL_ERR_VALUE;
                    word |= c << shift_of(j);
                }
                out[(n * blocks + b) * 16 + place_of(w)] = word;
            }
        }
    }
    return TL_OK;
}

tl_status tl_unpack_4bit(const uint32_t* packed, int64_t N, int64_t K, uint8_t* codes)
{
    using namespace tl;
    if (!packed || !codes) return TL_ERR_NULL;
    if (!product_ok(1, N, K)) return TL_ERR_SHAPE;
    const int64_t blocks = (K + 127) / 128;
    for (int64_t n = 0; n < N; ++n)
        for (int64_t k = 0; k < K; ++k) codes[n * K + k] = packed[(n * blocks + k / 128) * 16 + place_of(int(k % 128 / 8))] >> shift_of(int(k % 8)) & 15u;
    return TL_OK;
}

tl_status tl_gemm_4bit(const tl_gemm_4bit_job* job, void* stream)
{
    using namespace tl;
    if (!job) return TL_ERR_NULL;
    const tl_gemm_4bit_job& j = *job;
    if (!j.x || !j.Wpacked || !j.scales || !j.y) return TL_ERR_NULL;
    if (!product_ok(j.M, j.N, j.K) || j.N >= (int64_t(1) << 24) || j.K >= (int64_t(1) << 20) || !group_ok(j.group)) return TL_ERR_SHAPE;
    if (code_of(j.y_real) != TL_REAL_FP16 && code_of(j.y_real) != TL_REAL_FP32) return TL_ERR_UNSUPPORTED;
    if (!aligned(j.x, 16) || !aligned(j.Wpacked, 16) || !aligned(j.scales, 16) || !aligned(j.zeros, 16) || !aligned(j.y, 16)) return TL_ERR_ALIGN;
    const Gemm4Desc d{static_cast<const _Float16*>(j.x), static_cast<const uint32_t*>(j.Wpacked), static_cast<const _Float16*>(j.scales),
                      static_cast<const uint8_t*>(j.zeros), j.y, j.M, j.N, j.K, j.group, j.y_real == TL_REAL_FP32, 0};
    return from_hip(launch_gemm4(d, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
