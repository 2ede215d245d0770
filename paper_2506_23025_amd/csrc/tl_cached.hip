// Attention over the paged 8-bit cache: the plain kernel.  One wave per query row and head, 64 keys at a time: a lane takes a key for the
// scores, and a dimension (two beyond 64) for the sum over values.
#include "tl_attn.hpp"

namespace tl {
namespace {

template <bool FP8>
__device__ inline float value_of(uint32_t code)
{
    if constexpr (FP8) return __builtin_amdgcn_cvt_f32_fp8(int(code), 0);
    else return float(int(int8_t(code)));
}

template <bool FP8>
__global__ __launch_bounds__(64) void cached_kernel(CachedArgs a)
{
    const int lane = threadIdx.x, row = blockIdx.x, h = blockIdx.y, g = h / a.group;
    int s = row;
    if (a.b.start) {
        // the sequence of a row: the last that begins at or before it and is not empty
        int lo = 0, hi = a.b.seqs;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.b.start[mid] <= row) lo = mid; else hi = mid;
        }
        s = lo;
    }
    const Span sp = span(a.b, s);
    if (row < sp.first || row >= sp.first + sp.n) return;
    const int past = cached_of(a.b, s), dim = a.c.dim, chunks = dim >> 4;
    _Float16* out = a.out.p + int64_t(row) * a.out.token + int64_t(h) * a.out.head;
    const int64_t len = past < 0 ? 0 : int64_t(past) + (row - sp.first) + 1;
    __shared__ float q[128], p[64];
    for (int d = lane; d < dim; d += 64) q[d] = float(a.q.p[int64_t(row) * a.q.token + int64_t(h) * a.q.head + d]);
    __syncthreads();
    float m = -__builtin_inff(), l = 0.0f, o0 = 0.0f, o1 = 0.0f;
    const int blocks = 1 << a.c.page_shift;
    for (int64_t t0 = 0; t0 < len; t0 += 64) {
        const int64_t t = t0 + lane;
        const int page = t < len ? page_of(a.c, s, t >> 4) : -1;
        float x = -__builtin_inff();
        if (page >= 0) {
            const int64_t block = (int64_t(page) * a.c.kv_heads + g) * blocks + ((t >> 4) & (blocks - 1));
            const uint8_t* k = a.c.k + block * 16 * dim;
            const int i = int(t & 15);
            float sum = 0.0f;
            for (int d = 0; d < dim; ++d) sum += q[d] * value_of<FP8>(k[((i >> 2) * chunks + (d >> 4)) * 64 + (i & 3) * 16 + (d & 15)]);
            x = sum * (a.c.ks[block] * a.scale);
        }
        float mx = x;
        for (int k = 32; k; k >>= 1) mx = fmaxf(mx, __shfl_xor(mx, k));
        const float now = fmaxf(m, mx), base = now == -__builtin_inff() ? 0.0f : now;
        const float r = exp2f(m - base), e = page >= 0 ? exp2f(x - base) : 0.0f;
        float sum = e;
        for (int k = 32; k; k >>= 1) sum += __shfl_xor(sum, k);
        m = now;
        l = l * r + sum;
        o0 *= r;
        o1 *= r;
        __syncthreads();
        p[lane] = e;
        __syncthreads();
        for (int i = 0; i < 64 && t0 + i < len; ++i) {
            const int page_i = page_of(a.c, s, (t0 + i) >> 4);
            if (page_i < 0) continue;
            const int64_t block = (int64_t(page_i) * a.c.kv_heads + g) * blocks + (((t0 + i) >> 4) & (blocks - 1));
            const uint8_t* v = a.c.v + block * 16 * dim + ((t0 + i) & 15);
            const float w = p[i] * a.c.vs[block];
            if (lane < dim) o0 += w * value_of<FP8>(v[lane * 16]);
            if (lane + 64 < dim) o1 += w * value_of<FP8>(v[(lane + 64) * 16]);
        }
    }
    const float f = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    if (lane < dim) out[lane] = _Float16(o0 * f);
    if (lane + 64 < dim) out[lane + 64] = _Float16(o1 * f);
}

}  // namespace

size_t cached_workspace(int64_t, int64_t, int64_t, int64_t, int64_t) { return 16; }

hipError_t launch_cached(const CachedArgs& a, int64_t, hipStream_t s)
{
    const dim3 grid(unsigned(a.b.tokens), unsigned(a.q_heads));
    if (a.c.fp8) cached_kernel<true><<<grid, 64, 0, s>>>(a);
    else cached_kernel<false><<<grid, 64, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace tl
