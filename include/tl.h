/*
 * tl.h -- C ABI of the ternary-linear library for MI355X (gfx950).
 *
 * The library computes the inference form of the ternary linear layer of
 * Spectra-1.1 (arXiv 2506.23025):
 *
 *     Y = X * (gamma * What)^T          (paper App. B, "Inference", steps 1-3)
 *
 * with X fp16 [M][K], What in {-1,0,+1} [N][K] kept in one of the packed forms
 * of paper Sec. 3 and a single fp16 scale gamma per matrix (paper Sec. 2.1).
 * Accumulation is fp32 and the output is fp16 with round-to-nearest-even
 * (paper App. G, "Precision-Preserving Accumulation").
 *
 * Conventions shared by every entry point
 *   - All functions return a tl_status and never throw, abort or print.
 *   - "host" pointers are ordinary CPU memory; "device" pointers are HBM
 *     addresses valid on the current HIP device.  The caller owns every
 *     buffer; the library allocates nothing.  The only state it keeps between calls is
 *     a set of once-per-device flags that record that a kernel's launch attribute (its
 *     dynamic-LDS limit) has been set; tl_init sets them all.  Results never depend on it.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     Device entry points only enqueue work on that stream and return; they
 *     never synchronise.  Errors reported by the launch come back as
 *     TL_ERR_HIP.
 *   - Matrices are dense row-major.  Packed weights are row-major too: row n
 *     occupies tl_row_stride_bytes(fmt, K) bytes starting at
 *     n * tl_row_stride_bytes(fmt, K).
 */
#ifndef TL_H_
#define TL_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum tl_status {
    TL_OK = 0,
    TL_ERR_NULL = 1,        /* a required pointer is NULL                         */
    TL_ERR_SHAPE = 2,       /* M, N or K < 1, or a size product overflows          */
    TL_ERR_VALUE = 3,       /* weight outside {-1,0,1}, or an invalid packed code  */
    TL_ERR_ALIGN = 4,       /* device pointer not 16-byte aligned                  */
    TL_ERR_UNSUPPORTED = 5, /* unknown format / path, or path cannot run the shape */
    TL_ERR_HIP = 6          /* the HIP runtime reported an error on launch         */
} tl_status;

typedef enum tl_format {
    TL_FMT_2BIT = 0,   /* paper Sec. 3.1 with k = 16 digits per 32-bit word      */
    TL_FMT_1P6BIT = 1, /* 5 trits per byte, plain base 3 (see tl_pack_1p6bit)    */
    TL_FMT_1P6BIT_FX = 2, /* 5 trits per byte, the fixed-point code as the paper prints it
                            (see tl_pack_1p6bit_fx); same row geometry as TL_FMT_1P6BIT */
    TL_FMT_INT_RANGE_ = 0x7fffffff /* not a format: makes every non-negative int a value the type
                            can hold, so that an unknown code is reported, not undefined */
} tl_format;

/* Kernel choice for tl_ternary_gemm_path.  AUTO is what tl_ternary_gemm uses. */
typedef enum tl_path {
    TL_PATH_AUTO = 0,
    TL_PATH_GENERIC = 1, /* any M, N, K: forced, the plain VALU kernel; as the choice named by
                            tl_ternary_gemm_which, that or the tiled kernel's form for odd K */
    TL_PATH_GEMV = 2,    /* weight-streaming small-M kernel: M <= 16 per pass     */
    TL_PATH_MFMA = 3,    /* tiled fp16 MFMA kernel for many rows                 */
    TL_PATH_INT_RANGE_ = 0x7fffffff /* not a path (see TL_FMT_INT_RANGE_)         */
} tl_path;

/* Human-readable name of a status code (static storage, never NULL). */
const char* tl_status_str(tl_status s);

/*
 * Bytes from the start of one packed row to the next.
 *   TL_FMT_2BIT  : 4 * ceil(K / 16)                  (one uint32 per 16 weights)
 *   TL_FMT_1P6BIT: ceil(K / 5) rounded up to 16      (one byte per 5 weights;
 *                  the bytes after the last code byte are zero and never decoded)
 * Returns 0 for K < 1 or an unknown format.
 */
size_t tl_row_stride_bytes(tl_format fmt, int64_t K);

/* N * tl_row_stride_bytes(fmt, K); 0 on bad arguments. */
size_t tl_packed_bytes(tl_format fmt, int64_t N, int64_t K);

/*
 * Ternarisation of a trained weight matrix, paper App. B "Forward Pass":
 *   gamma = eps + mean |W_ij|,   What_ij = round(min(max(W_ij / gamma, -1), 1)).
 * The mean and the quotient are taken in fp64; round is round-half-to-even (the paper does
 * not say which; ties have measure zero for trained weights).  Per tensor only.
 *   W     host, float [N][K] row-major, finite
 *   What  host, int8 [N][K], written with values in {-1,0,1} (ready for tl_pack_*)
 *   gamma            if not NULL: the scale as computed (fp64)
 *   gamma_fp16_bits  if not NULL: the same rounded to fp16 (round to nearest even), the
 *                    form tl_ternary_gemm takes
 * TL_ERR_VALUE if W holds a NaN or an infinity, or eps is negative or not finite.
 */
tl_status tl_quantize(const float* W, int64_t N, int64_t K, double eps, int8_t* What,
                      double* gamma, uint16_t* gamma_fp16_bits);

/*
 * 2-bit packing P of paper Sec. 3.1 with k = 16: digit d' = w + 1 in {0,1,2};
 * word i of a row holds weights 16i .. 16i+15, weight 16i+j in bits [2j+1:2j].
 * A short last word is filled with weight 0 (digit 1), as the paper prescribes.
 *   W   host, int8 [N][K] row-major, every value in {-1,0,1}
 *   out host, uint32 [N][ceil(K/16)], written completely
 * TL_ERR_VALUE if any weight is outside {-1,0,1} (out is then unspecified).
 */
tl_status tl_pack_2bit(const int8_t* W, int64_t N, int64_t K, uint32_t* out);

/*
 * 1.6-bit packing: the base-3 block code of paper Sec. 3.2 (k = 5 digits in one
 * byte) in its plain, unscaled little-endian form: byte b of a row holds weights
 * 5b .. 5b+4 as sum_i (w[5b+i] + 1) * 3^i, a value in [0, 242].  Missing weights
 * of the last byte count as 0 (digit 1).  Rows are tl_row_stride_bytes apart and
 * the stride padding is written as zero.
 *   W   host, int8 [N][K];  out host, uint8 [N][stride]
 */
tl_status tl_pack_1p6bit(const int8_t* W, int64_t N, int64_t K, uint8_t* out);

/*
 * The fixed-point 1.6-bit code exactly as printed in paper Sec. 3.2 / App. E
 * (k = 5, p = 8): digits big-endian, Nval = sum_j d'_j 3^(4-j), byte =
 * floor((Nval * 256 + 242) / 243).  Same row geometry as tl_pack_1p6bit.
 * Decoded by tl_unpack_1p6bit_fx with the multiply-by-3 digit extraction of
 * paper App. F, Alg. 1 (on the GPU: tl_unpack_dev / tl_ternary_gemm_1p6_fx with
 * TL_FMT_1P6BIT_FX).
 */
tl_status tl_pack_1p6bit_fx(const int8_t* W, int64_t N, int64_t K, uint8_t* out);
tl_status tl_unpack_1p6bit_fx(const uint8_t* packed, int64_t N, int64_t K, int8_t* W_out);

/*
 * Unpacking U (paper Sec. 3.1 "Unpacking/Decoding"; Sec. 3.2 for base 3) on the
 * host.  packed: host, layout as written by the packers.  W_out: host int8
 * [N][K].  TL_ERR_VALUE on a 2-bit code 3 or a 1.6-bit byte > 242.
 */
tl_status tl_unpack(tl_format fmt, const void* packed, int64_t N, int64_t K, int8_t* W_out);

/*
 * The same decode on the GPU: packed and W_out are device pointers.  Invalid
 * codes are not reported; a 2-bit code 3 decodes to +2 and a byte > 242 to the
 * digits of its value modulo 243.  Exists so that the device decode can be
 * compared byte for byte with the host one.
 */
tl_status tl_unpack_dev(tl_format fmt, const void* packed, int64_t N, int64_t K,
                        int8_t* W_out, void* stream);

/*
 * y[m][n] = fp16_rne( float(gamma) * sum_k x[m][k] * w[n][k] ),  fp32 accumulation.
 *   x       device, fp16 [M][K] row-major, 16-byte aligned
 *   Wpacked device, TL_FMT_2BIT layout, 16-byte aligned
 *   gamma_fp16_bits  the per-matrix scale as raw IEEE binary16 bits
 *   y       device, fp16 [M][N] row-major, 16-byte aligned; fully overwritten
 * Activations are expected to be finite.  A NaN in row m of x makes row m of y NaN (no other
 * row); an infinity in row m makes that row NaN where the exact result would be +-infinity,
 * because the fast kernels compute sum (w + 1) x - sum x (Sec. 3.1 stores w + 1).
 * Any M, N, K >= 1 is accepted; the library picks the kernel from the shape
 * (small M: weight-streaming kernel; large M: tiled matrix-core kernel; K that is no
 * multiple of 64: the streaming or the tiled kernel's form for such rows, or the generic kernel).  Results are deterministic:
 * no atomics, fixed reduction order.  Behaviour on a 2-bit code 3 is memory-safe
 * but otherwise unspecified.
 */
tl_status tl_ternary_gemm(const void* x, const void* Wpacked, uint16_t gamma_fp16_bits,
                          void* y, int64_t M, int64_t N, int64_t K, void* stream);

/*
 * Optional.  Prepares every kernel of the library on the current HIP device (their limits for
 * dynamically sized LDS) so that no later call has to: without it each kernel instance does
 * this the first time it is launched.  Call it once per device, e.g. before capturing the
 * library's calls into a HIP graph.  Idempotent; allocates nothing; TL_ERR_HIP if the runtime
 * refuses.
 */
tl_status tl_init(void);

/*
 * The kernel tl_ternary_gemm (TL_PATH_AUTO) runs for a shape: TL_PATH_GEMV, TL_PATH_MFMA or
 * TL_PATH_GENERIC (K no multiple of 64: the any-shape kernels, i.e. the generic kernel or the streaming or
 * tiled kernel's form for odd K); TL_PATH_AUTO (0) if M, N or K is not a valid size.  A pure function of the
 * three numbers (host side, touches no GPU): the library's cost models of its two fast
 * kernels decide between them where both can run the shape.
 */
tl_path tl_ternary_gemm_which(int64_t M, int64_t N, int64_t K);

/* Same, with the kernel forced.  TL_ERR_UNSUPPORTED if `path` cannot run the shape. */
tl_status tl_ternary_gemm_path(const void* x, const void* Wpacked, uint16_t gamma_fp16_bits,
                               void* y, int64_t M, int64_t N, int64_t K, void* stream,
                               tl_path path);

/*
 * Several independent products in one call: the linears of a transformer block (the unit
 * the paper's kernel benchmark is quoted on, App. G "performance benchmark"), or any list
 * of (x, W, gamma, y).  Each job has the contract of tl_ternary_gemm.  No job reads what
 * another writes, and jobs must not alias
 * each other's outputs; they are enqueued in as few kernel launches as possible (jobs that
 * go to the small-M kernel share launches, 32 blocks of 16 or 32 activation rows per launch; a
 * job of many rows runs as tl_ternary_gemm would run it where that is faster) and
 * may run concurrently.  `jobs` is host memory, read before the call returns.
 */
typedef struct tl_gemm_job {
    const void* x;            /* device, fp16 [M][K]                */
    const void* Wpacked;      /* device, TL_FMT_2BIT                */
    void* y;                  /* device, fp16 [M][N]                */
    int64_t M, N, K;
    uint16_t gamma_fp16_bits;
} tl_gemm_job;

tl_status tl_ternary_gemm_grouped(const tl_gemm_job* jobs, int64_t count, void* stream);

/* Same contract for weights in the TL_FMT_1P6BIT layout of tl_pack_1p6bit. */
tl_status tl_ternary_gemm_1p6(const void* x, const void* Wpacked, uint16_t gamma_fp16_bits,
                              void* y, int64_t M, int64_t N, int64_t K, void* stream);

/*
 * Same contract for weights in the TL_FMT_1P6BIT_FX layout of tl_pack_1p6bit_fx: the
 * 1.6-bit code of paper Sec. 3.2 as printed, decoded on the GPU by the multiply-by-3 digit
 * extraction of App. F, Alg. 1 (the paper leaves a GPU kernel for this format as future
 * work, Sec. 3.3 "Limitations").
 */
tl_status tl_ternary_gemm_1p6_fx(const void* x, const void* Wpacked, uint16_t gamma_fp16_bits,
                                 void* y, int64_t M, int64_t N, int64_t K, void* stream);

/*
 * The same product with one fp16 scale per group of `group` consecutive weights along K and
 * per output row, in place of the single gamma:
 *     y[m][n] = sum_g scales[g][n] * ( sum_{k in group g} x[m][k] * w[n][k] )
 * (paper Sec. 3.3, CPU inference: the 2-bit block format keeps one fp16 scale per block of
 * 256 weights; GPU kernel appendix: the dequantised fragments are scaled by quantisation
 * scales held in a separate buffer).  `scales` is a device pointer to fp16
 * [ceil(K / group)][N], 16-byte aligned; the last group may be short.  x, Wpacked (2-bit
 * format), y, stream, accumulation and rounding as for tl_ternary_gemm.  `group` must be a
 * multiple of 16 (TL_ERR_SHAPE otherwise).  Scales are expected to be finite: an infinite one makes
 * the outputs of its column infinite or NaN, a NaN makes them NaN, and neither shows in another column.
 * Few activation rows, N % 4 == 0 and group % 64 == 0, or % 32 where K % 64 == 0, run in the
 * weight-streaming small-M kernel (M in blocks of 16 rows; the larger the power of two in `group`, up to
 * 256, the faster), the rest in the tiled kernel, except where so few rows make the generic kernel the
 * faster one.
 * Nothing is allocated; the call is asynchronous on `stream`.
 */
tl_status tl_ternary_gemm_gs(const void* x, const void* Wpacked, const void* scales, int64_t group,
                             void* y, int64_t M, int64_t N, int64_t K, void* stream);

/*
 * tl_ternary_gemm_grouped for the other two weight forms: several independent products in one
 * call, enqueued in as few kernel launches as possible (the launch costs as much as streaming
 * several megabytes, and the paper's kernel benchmark is quoted on all linears of a block,
 * App. G).  Jobs must not alias each other's outputs; `jobs` is host memory, read before the
 * call returns; each job has the contract of the single call it stands for.
 *
 * tl_ternary_gemm_1p6_grouped: weights in the 1.6-bit layout (Sec. 3.2), all jobs in the same
 * byte code: `format` is TL_FMT_1P6BIT (tl_pack_1p6bit) or TL_FMT_1P6BIT_FX (tl_pack_1p6bit_fx),
 * anything else is TL_ERR_VALUE.  Jobs with 8 <= K <= 4800 share launches (32 blocks
 * of 16 activation rows per launch) unless they have so many rows that a call of their own is faster, or more
 * than 16 and a K below 64 that is no multiple of 8; the others run as tl_ternary_gemm_1p6 / _fx would run them.
 */
tl_status tl_ternary_gemm_1p6_grouped(const tl_gemm_job* jobs, int64_t count, tl_format format,
                                      void* stream);

/*
 * tl_ternary_gemm_gs_grouped: 2-bit weights with per-group scales (Sec. 3.3; App. G), one group
 * size per job.  Jobs that tl_ternary_gemm_gs would run in the weight-streaming kernel share
 * launches (groups that are multiples of 256 weights among themselves, and so other multiples of 128, of
 * 64 and of 32) unless they have so many rows that a call of their own is faster; the others run one by one.
 */
typedef struct tl_gemm_gs_job {
    const void* x;            /* device, fp16 [M][K]                         */
    const void* Wpacked;      /* device, TL_FMT_2BIT                         */
    const void* scales;       /* device, fp16 [ceil(K / group)][N]           */
    void* y;                  /* device, fp16 [M][N]                         */
    int64_t M, N, K;
    int64_t group;            /* weights per scale along K, multiple of 16   */
} tl_gemm_gs_job;

tl_status tl_ternary_gemm_gs_grouped(const tl_gemm_gs_job* jobs, int64_t count, void* stream);

/*
 * ---- The attention of a block: positions, an 8-bit cache in pages, attention over it and over whole prompts ----
 *
 * What stands between the QKV and the O projection of a transformer block whose linears are the products above.  All
 * activations are fp16; softmax, sums and scales are fp32.
 *
 * A tensor of heads: element (token t, head h, dimension d) is the fp16 at ptr + t * token_stride + h * head_stride + d,
 * strides in elements, multiples of 8, not negative, below 2^24 from token to token and 2^40 from head to head; ptr 16-byte aligned.  So query, key and value may lie side by
 * side in the rows that one QKV product writes.
 */
typedef struct tl_heads {
    void* ptr;                /* device, fp16 */
    int64_t token_stride;
    int64_t head_stride;
} tl_heads;

/*
 * The tokens of a call: those of sequence s are rows seq_start[s] .. seq_start[s+1] - 1, and cached[s] tokens of the
 * sequence came before them, so that its token i stands at position cached[s] + i.  Both arrays are device memory and read
 * by the kernels, so a captured call serves every step.  seq_start does not decrease and lies in [0, tokens]; rows that no sequence has are neither read
 * nor written, and a sequence may have none.  cached[s] < 0 marks a sequence that is not in use: nothing of it
 * goes into the cache and its output rows are written as 0.
 */
typedef struct tl_batch {
    const int32_t* seq_start; /* device, [seqs + 1]; NULL: every sequence has one token (tokens == seqs)   */
    const int32_t* cached;    /* device, [seqs]; NULL: 0 for each                                          */
    int64_t seqs, tokens;     /* 1 <= seqs < 2^20; 0 <= tokens < 2^23 (0: the call does nothing)           */
} tl_batch;

/*
 * A cache of keys and values in 8 bits.  Pages of page_tokens tokens (16, 32, 64, ... 1024) hold all key heads; position p of
 * sequence s is in page page_table[s][p / page_tokens].  Sixteen tokens (positions 16 b .. 16 b + 15) and one head are a
 * block, which has one fp32 scale: a code stands for scale * code.  Codes are whole numbers in -127 .. 127
 * (TL_KV_INT8) or 8-bit floats with 4 exponent and 3 mantissa bits, largest 448 (TL_KV_FP8); the former are the nearer to
 * values of one size, the latter to values of many.
 *   k, v              device, [pages][kv_heads][page_tokens / 16][16 * head_dim] bytes, 16-byte aligned.  In a block, a
 *                     key's dimension d of token t is byte ((t / 4) * (head_dim / 16) + d / 16) * 64 + (t % 4) * 16 + d % 16, a value's
 *                     (d / 16) * 256 + (d % 16) * 16 + t: the orders in which the matrix instructions take them
 *   k_scale, v_scale  device, fp32 [pages][kv_heads][page_tokens / 16]
 *   page_table        device, int32 [seqs][pages_per_seq].  An entry outside [0, pages) stands for no page, and positions beyond
 *                     page_tokens * pages_per_seq have none: what would go there is dropped, and attention does not see it
 * Memory of pages need not be set to anything before they are used.  The cache belongs to the caller, and two calls
 * that write or read and write the same page have to be on one stream or ordered by the caller.
 */
typedef enum tl_kv_type {
    TL_KV_INT8 = 0,
    TL_KV_FP8 = 1,
    TL_KV_INT_RANGE_ = 0x7fffffff /* not a type (see TL_FMT_INT_RANGE_) */
} tl_kv_type;

typedef struct tl_kv_cache {
    void* k;
    void* v;
    float* k_scale;
    float* v_scale;
    const int32_t* page_table;
    int64_t pages, page_tokens, pages_per_seq;
    int64_t kv_heads, head_dim;
    tl_kv_type type;
} tl_kv_cache;

/*
 * Rotary positions.  Of each head the first rot_dim dimensions (even, at most head_dim) are turned in pairs,
 * (a, b) -> (a c - b s, a s + b c) with c = table[p][j] and s = table[p][rot_dim / 2 + j] for pair j at position p; the pair is
 * dimensions (j, rot_dim / 2 + j), or with `pairs` not 0 the neighbours (2 j, 2 j + 1).  Products and sums are fp32, each rounded by itself.
 *   table   device, fp32 [positions][rot_dim], 4-byte aligned (tl_rope_table fills one on the host).  A position that it does not
 *           reach gives NaN
 */
typedef struct tl_rope {
    const float* table;
    int64_t positions, rot_dim;
    int32_t pairs;
} tl_rope;

/*
 * Fills a host table for tl_rope: pair j turns by p * f_j with f_j = base^(-2 j / rot_dim), computed in fp64.  For contexts longer
 * than a model was trained on, `scaling` (NULL: none) changes the frequencies:
 *   TL_ROPE_LINEAR    f_j / factor
 *   TL_ROPE_BY_PARTS  a pair that turns t = trained * f_j / (2 pi) times over the trained length keeps f_j if t >= high, gets
 *                     f_j / factor if t <= low, and between them the mean of both weighted by (t - low) / (high - low)
 * and cosines and sines are multiplied by `magnitude`.  TL_ERR_SHAPE for positions or rot_dim < 1 or an odd rot_dim,
 * TL_ERR_VALUE for a base, factor or magnitude that is not positive and finite, or a range that is none, TL_ERR_UNSUPPORTED for an unknown kind.
 */
typedef enum tl_rope_kind {
    TL_ROPE_PLAIN = 0,
    TL_ROPE_LINEAR = 1,
    TL_ROPE_BY_PARTS = 2,
    TL_ROPE_INT_RANGE_ = 0x7fffffff /* not a kind (see TL_FMT_INT_RANGE_) */
} tl_rope_kind;

typedef struct tl_rope_scaling {
    tl_rope_kind kind;
    double factor;            /* TL_ROPE_LINEAR, TL_ROPE_BY_PARTS                  */
    double trained, low, high;/* TL_ROPE_BY_PARTS: 0 <= low < high, trained > 0     */
    double magnitude;
} tl_rope_scaling;

tl_status tl_rope_table(float* table, int64_t positions, int64_t rot_dim, double base, const tl_rope_scaling* scaling);

/*
 * Rotates the queries and keys of a call's tokens and puts keys and values into the cache.
 *   q, k, v        in; q_out, k_out: rotated and rounded to fp16 (ptr NULL: not wanted; they may be q and k themselves, with
 *                  the same strides, and may not overlap them otherwise).  q may have ptr NULL and q_heads 0, k and v ptr NULL where kv_heads is 0
 *   rope           NULL: no rotation
 *   cache          NULL: rotation alone (v is then not read); else kv_heads and head_dim as the cache has them
 *   head_dim       a multiple of 16 up to 128
 * What goes into the cache is coded from the fp32 rotated key and from the fp16 value.  A block's scale is that of the
 * tokens it holds before the call (0 if it holds none) or, if larger, the call's largest magnitude in it divided by 127 (448); where it grows, the
 * earlier codes are coded anew, round(code * (old scale / new scale)).  Places behind the last token keep what they hold.
 * A scale below 2^-80 becomes 0, and the call's codes in that block with it.
 * A block that takes a NaN or an infinity gets the scale NaN, and stands for NaN until its first token is written again.
 * Two sequences may not share a page that the call writes.
 */
typedef struct tl_append_job {
    tl_heads q, k, v, q_out, k_out;
    tl_batch batch;
    const tl_kv_cache* cache;
    const tl_rope* rope;
    int64_t q_heads, kv_heads, head_dim;
} tl_append_job;

tl_status tl_kv_append(const tl_append_job* job, void* stream);

/*
 * Attention of a call's tokens over the cache, which holds them already (tl_kv_append first): the query of token i of sequence s sees
 * positions 0 .. cached[s] + i, and
 *     out[t][h] = sum_p softmax_p(scale * q[t][h] . k[p][g]) v[p][g],   g = h / (q_heads / kv_heads).
 * A query that sees no position (all its pages missing) gives 0.  One with an infinity or a NaN in it gives NaN otherwise.
 * A block whose scale is NaN makes NaN of every query that sees a token of it, and of no other.
 *   q, out      q_heads heads of cache->head_dim dimensions; out may be q itself with the same strides, and may not overlap it otherwise
 *   scale       any sign; TL_ERR_VALUE where scale * log2(e) is not finite in fp32
 *   longest     an upper bound of cached[s] + the tokens of s over all sequences, 0 if not known: it spares the second
 *               launch that joins the parts of long sequences where none can be cut in parts.  Results are right also where it is exceeded
 *   workspace   device, 16-byte aligned, tl_attn_cached_workspace bytes at least; written and read within the call alone
 * Deterministic: no atomics, and the cuts depend on lengths and sizes alone.
 */
typedef struct tl_cached_job {
    tl_heads q, out;
    tl_batch batch;
    const tl_kv_cache* cache;
    int64_t q_heads;
    float scale;
    int64_t longest;
    void* workspace;
    size_t workspace_bytes;
} tl_cached_job;

size_t tl_attn_cached_workspace(int64_t seqs, int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t head_dim);
tl_status tl_attn_cached(const tl_cached_job* job, void* stream);

/*
 * Attention of whole prompts, causal: token i of a sequence sees tokens 0 .. i of the same sequence among this call's rows
 * (batch.cached is not read), with fp16 keys and values:
 *     out[t][h] = sum_j softmax_j(scale * q[t][h] . k[j][g]) v[j][g],   g = h / (q_heads / kv_heads).
 * head_dim is a multiple of 16 up to 128; (seqs + tokens / 32) * q_heads is below 2^24; scale as in tl_cached_job.  An infinity or a NaN in a key or value shows in the tokens that see it and in no others.  A token
 * whose scores are all -infinity gives NaN, and so does one with an infinity or a NaN in its query.  out may be
 * q itself with the same strides, and may not overlap q, k or v otherwise.  Deterministic.
 */
typedef struct tl_prompt_job {
    tl_heads q, k, v, out;
    tl_batch batch;
    int64_t q_heads, kv_heads, head_dim;
    float scale;
} tl_prompt_job;

tl_status tl_attn_prompt(const tl_prompt_job* job, void* stream);

/*
 * ---- Rows in 8 bits: the norms and gates of a block that make them, ternary products that take them ----
 *
 * Between its products a block adds to its residual, takes a norm of it, and weighs the up product by the gate.  Those steps can leave their rows in
 * 8 bits with a scale for each row, and the ternary products then run on whole numbers: exactly, with half the bytes of activations, and at twice
 * the matrix rate.
 *
 * Rows of numbers: element (row r, place d) at ptr + r * stride + d, fp16 unless said otherwise.  ptr is 16-byte aligned; the stride is in elements, a
 * multiple of 16 bytes, not negative and below 2^40; rows that a call writes are at least as far apart as they are long (one row alone: any stride).
 * Products write dense rows, and tl_gemm_4bit reads such: several rows of a product go straight into these calls, and theirs into it, where the number of places is a multiple of 8.
 */
typedef struct tl_rows {
    void* ptr;                /* device */
    int64_t stride;
} tl_rows;

/*
 * Rows of 8-bit codes, -127 .. 127: place d of row r stands for scales[r] * code.  In each block of 16 places, place 4 i + s is byte 4 s + i (i, s = 0 .. 3): the order
 * in which two bits of every byte of a packed word's bits meet them.  A row's last block is filled with 0; bytes behind it are
 * not written, and what they hold does not matter.
 *   codes    device, 16-byte aligned; rows are `stride` bytes apart, a multiple of 16 of at least ceil(places / 16) * 16 and below 2^24 (one row alone: any such multiple or 0)
 *   scales   device, fp32 [rows], 4-byte aligned
 * A row v becomes codes by its largest magnitude t: scale t / 127, code round(v * (127 / t)), quotients, product and rounding (to the nearest, ties
 * to even) each as IEEE fp32 has them.  With t below 2^-100 scale and codes are 0; with an infinity or a NaN in v the scale is NaN and the codes are 0.
 */
typedef struct tl_rows8 {
    int8_t* codes;
    float* scales;
    int64_t stride;
} tl_rows8;

typedef enum tl_real {
    TL_REAL_FP16 = 0,
    TL_REAL_FP32 = 1,
    TL_REAL_INT_RANGE_ = 0x7fffffff /* not a type (see TL_FMT_INT_RANGE_) */
} tl_real;

/*
 * The residual's addition and a root-mean-square norm:
 *     s = residual + x                         rounded to `real`, kept in sum
 *     v = (s * r) * weight,   r = 1 / sqrt(mean(s^2) + eps)
 *     y = v in fp16,  out = v in 8 bits
 * mean, root and quotient are taken in fp64 and r rounded to fp32; both products are fp32, each rounded by itself.
 *   x         fp16
 *   residual  `real`; ptr NULL: s = x, and sum is not written.  sum may be residual itself with the same stride, and x where real is TL_REAL_FP16; no other overlap with what
 *             is read, here and below
 *   sum       `real`; ptr NULL: not wanted
 *   weight    device, fp16 [dim], 16-byte aligned; NULL: 1
 *   y         ptr NULL: not wanted (it may be x with the same stride);  out: codes NULL: not wanted
 *   rows >= 0 below 2^31 (0: the call does nothing), 1 <= dim <= 65536, eps >= 0 and finite (a row of zeros with eps 0 gives NaN)
 * Deterministic.  TL_ERR_NULL where none of sum, y and out is wanted.
 */
typedef struct tl_norm_job {
    tl_rows x, residual, sum, y;
    tl_rows8 out;
    const void* weight;
    int64_t rows, dim;
    float eps;
    tl_real real;             /* of residual and sum */
} tl_norm_job;

tl_status tl_norm(const tl_norm_job* job, void* stream);

/*
 * The gate between the up and the down product, or (gate.ptr NULL) rows as they are, into fp16 and / or 8 bits:
 *     v = gate / (1 + exp(-gate)) * up         in fp64, rounded to fp32 once;   or v = up
 *     y = v in fp16,  out = v in 8 bits
 * gate and up may lie side by side in the rows that one product writes.  y may be gate or up with the same stride.  rows and dim as in tl_norm.  Deterministic.
 * TL_ERR_NULL where neither y nor out is wanted.
 */
typedef struct tl_gate_job {
    tl_rows gate, up, y;
    tl_rows8 out;
    int64_t rows, dim;
} tl_gate_job;

tl_status tl_gate(const tl_gate_job* job, void* stream);

/*
 * Ternary products over 8-bit rows:
 *     y[m][n] = fp16_rne( float(sum_k code[m][k] * w[n][k]) * (scale[m] * float(gamma)) ),
 * the sum exact (rounded once to fp32 where it is beyond 2^24), products fp32.  Wpacked, gamma and y as for tl_ternary_gemm; x: M rows of K places.  Any M as there, N and K
 * below 2^24.  A scale that is infinite or NaN shows in its row of y and in no other (0 codes with a scale of NaN give NaN).  Codes of -128 are taken as they are.  What a row's
 * bytes behind place K - 1 hold does not matter.  Deterministic: the sums are whole numbers.
 * tl_ternary_gemm_rows8_grouped: several independent products in one call, in as few launches as possible; jobs must not alias each other's
 * outputs; `jobs` is host memory, read before the call returns.
 */
typedef struct tl_gemm_rows8_job {
    tl_rows8 x;
    const void* Wpacked;      /* device, TL_FMT_2BIT   */
    void* y;                  /* device, fp16 [M][N]   */
    int64_t M, N, K;
    uint16_t gamma_fp16_bits;
} tl_gemm_rows8_job;

tl_status tl_ternary_gemm_rows8(const tl_gemm_rows8_job* job, void* stream);
tl_status tl_ternary_gemm_rows8_grouped(const tl_gemm_rows8_job* jobs, int64_t count, void* stream);

/*
 * ---- 4-bit weights with group scales: for the layers that ternary weights do not serve, the head first ----
 *
 * A weight is scales[g][n] * (c - z): code c in 0 .. 15, g = k / group, z = zeros[g][n] or 8.  The paper's 4-bit family keeps one
 * scale per 128 weights of a row (Sec. 3.3 compares with it).
 *
 * Packed form: a row's codes in blocks of 128 (the last filled with code 0), 16 words of 32 bits each.  Word w holds weights 8 w .. 8 w + 7 of the block
 * and stands at place 4 (w % 4) + w / 4; in it weight 2 j has bits 4 j .. 4 j + 3 and weight 2 j + 1 bits 4 j + 16 .. 4 j + 19: a lane's 16 bytes are its operands
 * of four matrix instructions, and one mask takes two neighbours.  Rows are tl_row_stride_4bit(K) = 64 ceil(K / 128) bytes apart (0 for K < 1).
 *
 * tl_quantize_4bit: codes of a trained matrix, host.  Without zeros scale = fp16(max|w| / 7) over the group and c = 8 + round(w / scale), held in 0 .. 15; with zeros
 * lo = min(0, w), hi = max(0, w), scale = fp16((hi - lo) / 15), z = round(-lo / scale), c = z + round(w / scale), both held in 0 .. 15.  Quotients in fp64, ties to even; a
 * scale of 0 gives codes 8 (z = 8).
 *   W host, float [N][K], finite;  codes host, uint8 [N][K];  scales host, fp16 bits [ceil(K / group)][N];  zeros host, uint8 of the same shape, or NULL
 * TL_ERR_VALUE if W holds a NaN or an infinity, or a group's scale is beyond fp16; group as for tl_gemm_4bit.
 * tl_pack_4bit (TL_ERR_VALUE on a code above 15), tl_unpack_4bit: host, codes uint8 [N][K].
 */
size_t tl_row_stride_4bit(int64_t K);
tl_status tl_quantize_4bit(const float* W, int64_t N, int64_t K, int64_t group, uint8_t* codes, uint16_t* scales_fp16_bits, uint8_t* zeros);
tl_status tl_pack_4bit(const uint8_t* codes, int64_t N, int64_t K, uint32_t* out);
tl_status tl_unpack_4bit(const uint32_t* packed, int64_t N, int64_t K, uint8_t* codes);

/*
 * y[m][n] = sum_g scales[g][n] * ( sum_{k in group g} x[m][k] * (c[n][k] - z[g][n]) ),  fp32 accumulation, rounded once to y's type.
 *   x        device, fp16 [M][K], 16-byte aligned
 *   Wpacked  device, packed form, 16-byte aligned
 *   scales   device, fp16 [ceil(K / group)][N], 16-byte aligned;  zeros: device, uint8 of the same shape, 16-byte aligned (any byte is taken as it is), or NULL
 *   y        device, fp16 or fp32 [M][N], 16-byte aligned
 *   group    a multiple of 32; the last group may be short
 * Any M >= 1, N below 2^24, K below 2^20; made for few rows (a pass over the weights serves up to 64).  A NaN or an infinity in row m of x shows in row m of y and in no other, one in a scale in its
 * column.  Deterministic: no atomics, fixed order.
 */
typedef struct tl_gemm_4bit_job {
    const void* x;
    const void* Wpacked;
    const void* scales;
    const void* zeros;
    void* y;
    int64_t M, N, K, group;
    tl_real y_real;
} tl_gemm_4bit_job;

tl_status tl_gemm_4bit(const tl_gemm_4bit_job* job, void* stream);

/*
 * Bandwidth calibration: a plain streaming copy dst[i] = src[i] of `bytes` bytes
 * (multiple of 16, both device pointers 16-byte aligned).  Not part of the
 * method; it gives the HBM counters and timers a kernel of known traffic.
 */
tl_status tl_probe_copy(void* dst, const void* src, size_t bytes, void* stream);

/*
 * Bandwidth ceiling: a streaming read of `bytes` bytes (multiple of 16, `src` a device
 * pointer, 16-byte aligned) that does nothing with them -- one launch, as many workgroups as
 * the buffer has 16 KB pieces.  No kernel that streams a weight matrix of that size once per
 * launch (Sec. 3.3: the memory-bound regime) can finish sooner; the benchmark times it beside
 * the GEMM kernels.  `sink` is a device pointer to 4 writable bytes, 4-byte aligned, written
 * only if the fold of all words read equals one particular value (it keeps the loads alive).
 * Not part of the method.
 */
tl_status tl_probe_read(const void* src, size_t bytes, void* sink, void* stream);

/*
 * Matrix-pipe ceiling for the large-batch regime (Sec. 3.3: beyond the critical batch the product
 * is compute-bound; App. G: the dequantised weights feed the matrix units): a kernel whose waves
 * do nothing but fp16 matrix instructions (v_mfma_f32_32x32x16_f16, 8 independent accumulators
 * per wave, two waves per SIMD of a 256-CU device) for `iters` rounds.  The operands are real data,
 * since what the chip sustains depends on it: activations read from `x` (device, fp16, x_elems >= 1
 * of them, reused cyclically) against ternary weights decoded to -1 / 0 / +1 from `Wpacked`
 * (device, 2-bit words, w_words >= 1).  `*flops` (host, may be NULL) receives the floating-point
 * operations of the launch; `sink` is a device pointer to 4 writable bytes (written only if the
 * fold of all sums equals one particular value).  Not part of the method: the benchmark times it
 * beside the large-M kernel.
 */
tl_status tl_probe_mfma(const void* x, int64_t x_elems, const void* Wpacked, int64_t w_words, int64_t iters,
                        void* sink, double* flops, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TL_H_ */
