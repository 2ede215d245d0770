// Causal attention over packed prompts: the plain kernel.  One wave per query row and head, 64 keys at a time.
#include "tl_attn.hpp"

namespace tl {
namespace {

__global__ __launch_bounds__(64) void prompt_kernel(PromptArgs a)
{
    const int lane = threadIdx.x, row = blockIdx.x, h = blockIdx.y, g = h / a.group, dim = a.dim;
    int s = row;
    if (a.b.start) {
        int lo = 0, hi = a.b.seqs;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.b.start[mid] <= row) lo = mid; else hi = mid;
        }
        s = lo;
    }
    const Span sp = span(a.b, s);
    if (row < sp.first || row >= sp.first + sp.n) return;
    __shared__ float q[128], p[64];
    for (int d = lane; d < dim; d += 64) q[d] = float(a.q.p[int64_t(row) * a.q.token + int64_t(h) * a.q.head + d]);
    __syncthreads();
    const _Float16* k = a.k.p + int64_t(sp.first) * a.k.token + int64_t(g) * a.k.head;
    const _Float16* v = a.v.p + int64_t(sp.first) * a.v.token + int64_t(g) * a.v.head;
    float m = -__builtin_inff(), l = 0.0f, o0 = 0.0f, o1 = 0.0f;
    const int len = row - sp.first + 1;
    for (int t0 = 0; t0 < len; t0 += 64) {
        const int t = t0 + lane;
        float x = -__builtin_inff();
        if (t < len) {
            float sum = 0.0f;
            for (int d = 0; d < dim; ++d) sum += q[d] * float(k[int64_t(t) * a.k.token + d]);
            x = sum * a.scale;
        }
        float mx = x;
        for (int i = 32; i; i >>= 1) mx = fmaxf(mx, __shfl_xor(mx, i));
        const float now = fmaxf(m, mx), base = now == -__builtin_inff() ? 0.0f : now;
        const float r = exp2f(m - base), e = t < len ? exp2f(x - base) : 0.0f;
        float sum = e;
        for (int i = 32; i; i >>= 1) sum += __shfl_xor(sum, i);
        m = now;
        l = l * r + sum;
        o0 *= r;
        o1 *= r;
        __syncthreads();
        p[lane] = e;
        __syncthreads();
        for (int i = 0; i < 64 && t0 + i < len; ++i) {
            const _Float16* vi = v + int64_t(t0 + i) * a.v.token;
            if (lane < dim) o0 += p[i] * float(vi[lane]);
            if (lane + 64 < dim) o1 += p[i] * float(vi[lane + 64]);
        }
    }
    const float f = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    _Float16* out = a.out.p + int64_t(row) * a.out.token + int64_t(h) * a.out.head;
    if (lane < dim) out[lane] = _Float16(o0 * f);
    if (lane + 64 < dim) out[lane + 64] = _Float16(o1 * f);
}

}  // namespace

hipError_t launch_prompt(const PromptArgs& a, hipStream_t s)
{
    const dim3 grid(unsigned(a.b.tokens), unsigned(a.q_heads));
    prompt_kernel<<<grid, 64, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace tl
