// What the kernels of the attention part share: their arguments and the look-up of a sequence.
#pragma once
#include "tl_internal.hpp"

namespace tl {

struct Heads {
    _Float16* p;
    int64_t token, head;                  // strides in elements
};

struct Batch {
    const int* start;                     // NULL: one token per sequence
    const int* cached;                    // NULL: 0
    int seqs, tokens;
};

struct Cache {
    uint8_t *k, *v;
    float *ks, *vs;
    const int* table;
    int64_t pages, pages_per_seq;
    int kv_heads, dim;
    int page_shift;                       // log2 of the blocks of 16 tokens in a page
    int fp8;
};

struct Rope {
    const float* table;                   // NULL: no rotation
    int64_t positions;
    int rot, pairs;
    int wide;                             // rows of the table and groups of 8 dimensions can be read 16 bytes at a time
};

struct AppendArgs {
    Heads q, k, v, q_out, k_out;
    Batch b;
    Cache c;                              // k == NULL: no cache
    Rope r;
    int q_heads, kv_heads, dim;
};

struct CachedArgs {
    Heads q, out;
    Batch b;
    Cache c;
    int q_heads, group;                   // query heads, and how many share a key head
    float scale;                          // times log2(e): the softmax works with powers of 2
    float* part;                          // workspace
};

struct PromptArgs {
    Heads q, k, v, out;
    Batch b;
    int q_heads, kv_heads, group, dim;
    float scale;
};

// Weights go into the second product in fp16, as powers of 2 relative to a running reference.  kSlack: log2 of how far a row's largest may pass its reference before that moves; kLift: log2 of what a weight at the
// reference is in fp16.  Their sum is what fp16 holds (up to 2^15); with the lift at that, a weight is off by 2^-11 of itself down to 2^-21 of the reference, and below by 2^-32 of it.
constexpr float kSlack = 8.0f, kLift = 7.0f;

hipError_t launch_append(const AppendArgs& a, hipStream_t s);
hipError_t launch_cached(const CachedArgs& a, int64_t longest, hipStream_t s);
size_t cached_workspace(int64_t seqs, int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t dim);
hipError_t launch_prompt(const PromptArgs& a, hipStream_t s);

// Rows [first, first + n) of sequence s, whatever the array holds.
struct Span { int first, n; };
__device__ inline Span span(const Batch& b, int s)
{
    if (!b.start) return {s, 1};
    int x = b.start[s], y = b.start[s + 1];
    x = x < 0 ? 0 : x > b.tokens ? b.tokens : x;
    y = y < x ? x : y > b.tokens ? b.tokens : y;
    return {x, y - x};
}

__device__ inline int cached_of(const Batch& b, int s) { return b.cached ? b.cached[s] : 0; }

// Work items of a call are numbered so that the host knows how many there can be without reading the lengths: sequence s has
// the items from start[s] / per + extra * s on, and needs no more than the next one's begin leaves it (`extra` = 1 where
// it needs ceil(n / per), 2 where its pieces of `per` may begin anywhere).
__device__ inline int item_base(const Batch& b, int s, int per, int extra)
{
    int x = b.start[s];
    x = x < 0 ? 0 : x > b.tokens ? b.tokens : x;
    return x / per + extra * s;
}

// The sequence that an item belongs to, and which of its items it is; {-1, 0} for none.  All lanes of the wave look at once: 64 places a round.
struct Item { int seq, i; };
__device__ inline Item find_item(const Batch& b, int item, int per, int extra)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = b.seqs;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, at = lo + lane * step;
        const bool before = at < hi && item_base(b, at, per, extra) <= item;
        const int n = __popcll(__ballot(before));
        if (n == 0) return {-1, 0};
        lo += (n - 1) * step;
        if (lo + step < hi) hi = lo + step;
    }
    const int base = item_base(b, lo, per, extra);
    if (base > item) return {-1, 0};
    return {lo, item - base};
}

// Page of a block of 16 tokens of sequence s, or -1.  Without a branch: lanes ask for different blocks, and matrix instructions have to find them all together.
__device__ inline int page_of(const Cache& c, int s, int64_t block)
{
    const int64_t i = block >> c.page_shift, last = c.pages_per_seq - 1;
    const int p = c.table[int64_t(s) * c.pages_per_seq + (i < last ? i : last)];
    return i <= last && p >= 0 && p < c.pages ? p : -1;
}

// The sum over the wave.
template <int CTRL, int ROWS>
__device__ inline int moved(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 15, true); }
__device__ inline int wave_sum(int x)
{
    x += moved<0x111, 15>(x);             // from the lane 1, 2, 4 and 8 before in the row of 16
    x += moved<0x112, 15>(x);
    x += moved<0x114, 15>(x);
    x += moved<0x118, 15>(x);
    x += moved<0x142, 10>(x);             // a row's last lane to the next row, rows 1 and 3
    x += moved<0x143, 12>(x);             // lane 31 to rows 2 and 3
    return __builtin_amdgcn_readlane(x, 63);
}

// A value that all lanes have, in a scalar register.
__device__ inline int same(int x) { return __builtin_amdgcn_readfirstlane(x); }

}  // namespace tl
