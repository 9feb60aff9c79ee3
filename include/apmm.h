/*
 * apmm.h - C ABI of the bipolar-INT arbitrary-precision GEMM library for MI355X (gfx950).
 *
 * The library computes C = A * W^T where A (M x K activations, p bits) and W (N x K
 * weights, q bits) hold bipolar-INT codes: bit i of a code contributes (2*bit - 1) * 2^i
 * (paper Sec. 3.1, Eq. 1), so an n-bit code u has the value 2u - (2^n - 1).
 * The operands are first decomposed into 1-bit planes, reassembled into 32-bit words
 * and concatenated into one buffer (paper Sec. 4.1, steps 1-3: apmm_pack_*); the GEMM
 * multiplies the planes and recovers C = sum_i sum_j 2^(i+j) * D_ij on chip, never in
 * global memory (paper Sec. 3.2 and Sec. 4.2: apmm_gemm).
 *
 * Conventions
 *  - Every data pointer is a DEVICE pointer owned by the caller.  The library allocates
 *    no device memory and keeps no state besides a thread-local error string.
 *  - `stream` is a hipStream_t passed as void* (NULL = the null stream).  All work is
 *    enqueued asynchronously on it; the call returns once the kernels are launched.
 *  - Argument errors are detected on the host before any launch and leave the outputs
 *    untouched.
 *  - Codes are one uint8 per element, row-major with K contiguous; only the low `bits`
 *    bits are significant, higher bits are ignored.
 *  - Packed buffers are opaque.  Their size is apmm_packed_bytes() for weights and
 *    apmm_packed_activation_bytes() for activations; the only contractual property is
 *    apmm_unpack*(apmm_pack_*(x)) == x on the low `bits` bits.  They must be
 *    16-byte aligned (any hipMalloc / PyTorch allocation is).
 *  - Unpacked codes and binary16 activations may lie at any address of their type's alignment.  Rows that do not start at whole
 *    aligned 4-byte words are read in such words: a call may read (never write, and never use) up to three bytes before the
 *    matrix and up to three after it, within the aligned words that hold its first and its last byte.
 */
#ifndef APMM_H
#define APMM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    APMM_OK = 0,
    APMM_ERR_INVALID_ARG = 1, /* null pointer, negative size, bits outside [1, 8], misaligned buffer */
    APMM_ERR_UNSUPPORTED = 2, /* valid request that no kernel in this build covers */
    APMM_ERR_OVERFLOW = 3,    /* K * (2^p - 1) * (2^q - 1) does not fit the 32-bit output */
    APMM_ERR_WORKSPACE = 4,   /* workspace missing or smaller than the call needs (apmm_gemm_from_codes) */
    APMM_ERR_HIP = 5          /* a HIP call failed; text in apmm_last_error() */
} apmm_status;

/* Kernel selection for apmm_gemm_ex.  apmm_gemm uses APMM_ALGO_AUTO. */
typedef enum {
    APMM_ALGO_AUTO = 0,
    APMM_ALGO_VALU_POPCOUNT = 1, /* plane pairs by XOR + popcount on the vector ALU, D_ij = K - 2*popc */
    APMM_ALGO_DECODE = 3,        /* small-M weight-streaming kernels: p, q <= 4 and M <= 64 (unpacked activation codes of 3 and
                                    4 bits: M <= 32) within the K bound of APMM_ALGO_MFMA_FP4, else M <= 16, q <= 4 and p not 3
                                    or 4; on the fp4 or int8 matrix operations, or XOR + popcount where that is faster or K is
                                    beyond the bound */
    APMM_ALGO_MFMA_FP4 = 4,      /* plane groups recombined to E2M1 codes in registers, f8f6f4 MFMA, exact fp32 accumulate
                                    (p, q <= 4 and 4 * roundup(K,512) * (2^p-1)(2^q-1) < 2^24); the large-tile kernel, every
                                    wave sweeping all of K */
    APMM_ALGO_DECODE_VALU = 5,   /* the XOR + popcount small-M kernel whatever the widths (M <= 16, q <= 4, p not 3 or 4):
                                    design B at decode shapes, for comparison */
    /* Ablation for the claim of paper Sec. 4.2 (p <= 2, q <= 4, same K bound as APMM_ALGO_MFMA_FP4); planes as +-1
       operands on the matrix unit: */
    APMM_ALGO_PLANE_PAIRS_GLOBAL = 6, /* the scheme the paper argues against: one plane pair per workgroup, its 32-bit
                                    product D_ij to global memory, then a pass that shifts and adds them into C.
                                    Needs `workspace` of p * q * M * N * 4 bytes (16-byte aligned), else
                                    APMM_ERR_WORKSPACE */
    APMM_ALGO_PLANES_REGISTERS = 7, /* one tile per workgroup, an accumulator per plane pair, shift-and-add in registers
                                    (the paper's recovery-oriented scheme) */
    APMM_ALGO_MFMA_KSPLIT = 8    /* APMM_ALGO_MFMA_FP4 with the K partition of paper Sec. 4.2 taken across the four waves of
                                    a workgroup as well: every wave holds the whole workgroup tile for a quarter of K, the
                                    partial tiles are added in LDS (chosen by AUTO for outputs of one round of tiles and long K) */
} apmm_algo;

/* Bytes of the packed form of a rows x K operand of `bits`-bit codes (paper Sec. 4.1:
 * `bits` bits per element in 32-bit words, concatenated, plus one int32 per row).  Rows are padded
 * to a multiple of 32 and K to a multiple of 512.  Returns 0 for invalid arguments. */
size_t apmm_packed_bytes(int64_t rows, int64_t K, int bits);

/* Bytes of the packed form of M x K activations of p bits.  Equal to apmm_packed_bytes(M, K, p) except
 * for p = 3 and 4, whose codes are stored as 6-bit fields, the matrix unit's own operand form, so that
 * the GEMM needs no expansion for them. */
size_t apmm_packed_activation_bytes(int64_t M, int64_t K, int p);

/* Bytes of scratch apmm_gemm needs for this problem (may be 0). */
size_t apmm_workspace_bytes(int64_t M, int64_t N, int64_t K, int p, int q);

/* Paper Sec. 4.1 (matrix decomposition and reassembly) for the weight matrix.
 *   w_codes  : device, N x K uint8 codes, row-major.
 *   w_packed : device, apmm_packed_bytes(N, K, q) bytes, written entirely.
 * N == 0 is allowed (nothing is done).  K must be >= 1. */
apmm_status apmm_pack_weights(const uint8_t *w_codes, int64_t N, int64_t K, int q,
                              void *w_packed, void *stream);

/* Same transform for the activation matrix (M x K codes of p bits); meant to run online,
 * directly before apmm_gemm on the same stream.  a_packed: apmm_packed_activation_bytes(M, K, p) bytes. */
apmm_status apmm_pack_activations(const uint8_t *a_codes, int64_t M, int64_t K, int p,
                                  void *a_packed, void *stream);

/* Paper Sec. 3.1 (the feature matrix is quantised onto the symmetric bipolar-INT grid) fused with the
 * packing of Sec. 4.1, for activations that arrive as binary16 numbers: one pass instead of writing and
 * re-reading one code byte per element.  Per row (token) m:
 *   a_scale[m] = max_k |x[m][k]| / (2^p - 1), correctly rounded to binary16 (nearest, ties to even)
 *   code       = (v + 2^p - 1) / 2, v = the odd integer of [-(2^p - 1), 2^p - 1] nearest to x / a_scale[m],
 *                the upper one on a tie
 * decided as in exact arithmetic on the binary16 values (an element exactly on a cell border
 * x = 2 c a_scale[m] always lands in the upper cell); a row whose scale rounds to zero gets the code of +1
 * everywhere.  The result is the packed operand apmm_pack_activations would give
 * for those codes, and a_scale is the per-token scale for apmm_gemm's fp16 epilogue.
 *   x_f16    : device, M x K binary16 bit patterns, row-major, finite values
 *   a_packed : device, apmm_packed_activation_bytes(M, K, p) bytes, written entirely
 *   a_scale  : device, M binary16 bit patterns, written */
apmm_status apmm_quantize_pack_activations(const uint16_t *x_f16, int64_t M, int64_t K, int p,
                                           void *a_packed, uint16_t *a_scale, void *stream);

/* Inverse of apmm_pack_weights (test aid): writes rows x K uint8 codes. */
apmm_status apmm_unpack(const void *packed, int64_t rows, int64_t K, int bits,
                        uint8_t *codes, void *stream);
/* Inverse of apmm_pack_activations (test aid): writes M x K uint8 codes. */
apmm_status apmm_unpack_activations(const void *a_packed, int64_t M, int64_t K, int p,
                                    uint8_t *codes, void *stream);

/* Paper Sec. 3.2 (bit-wise MatMul reconstitution) with the recovery of Sec. 4.2 kept on chip.
 *   a_packed : device, packed M x K activations of p bits (from apmm_pack_activations)
 *   w_packed : device, packed N x K weights of q bits     (from apmm_pack_weights)
 *   c_i32    : device, M x N row-major int32 result, or NULL
 *   c_f16    : device, M x N row-major IEEE binary16 bit patterns of
 *              C[m][n] * a_scale[m] * w_scale[n] (product in fp32, one rounding to
 *              nearest-even at the end; a product beyond the binary16 range, |x| >= 65520,
 *              becomes an infinity of its sign, as IEEE 754 rounding has it), or NULL
 *   w_scale  : device, N binary16 per-output-channel scales, or NULL (= 1)
 *   a_scale  : device, M binary16 per-token scales, or NULL (= 1)
 *   workspace: device scratch of at least apmm_workspace_bytes() bytes (may be NULL if 0; only
 *              APMM_ALGO_PLANE_PAIRS_GLOBAL of apmm_gemm_ex uses one)
 * At least one of c_i32 / c_f16 must be non-NULL.  M == 0 or N == 0 returns APMM_OK
 * without a launch.  Returns APMM_ERR_OVERFLOW if roundup(K,512)*(2^p-1)*(2^q-1) > INT32_MAX. */
apmm_status apmm_gemm(int64_t M, int64_t N, int64_t K, int p, int q,
                      const void *a_packed, const void *w_packed,
                      int32_t *c_i32, uint16_t *c_f16,
                      const uint16_t *w_scale, const uint16_t *a_scale,
                      void *workspace, size_t workspace_bytes, void *stream);

/* apmm_gemm with an explicit kernel choice (used to compare the two designs).
 * Returns APMM_ERR_UNSUPPORTED if `algo` does not cover the request. */
apmm_status apmm_gemm_ex(int64_t M, int64_t N, int64_t K, int p, int q,
                         const void *a_packed, const void *w_packed,
                         int32_t *c_i32, uint16_t *c_f16,
                         const uint16_t *w_scale, const uint16_t *a_scale,
                         void *workspace, size_t workspace_bytes, void *stream,
                         int algo);

/* apmm_gemm taking the activation codes as they are: the preprocessing of paper Sec. 4.1 (decomposition,
 * reassembly, concatenation) for the activations and the bit-wise MatMul of Sec. 3.2 in one call, as an
 * inference engine meets them (Sec. 5.2: the activations of a layer are produced online).  `a_codes` is
 * the device M x K row-major uint8 matrix that apmm_pack_activations would take (bits above p are
 * ignored, no alignment needed).  Result and all other arguments as in apmm_gemm.
 *   - For a few tokens the small-M kernels regroup the codes into the packed form on their way into
 *     on-chip memory: one launch, no packed buffer.  The separate packing launch costs as much as such a
 *     GEMM.  Taken for shapes of APMM_ALGO_DECODE when M <= 16 (3- and 4-bit activations: M <= 8) or M * N <=
 *     65536, and, with a workspace, for every other pair of widths with a code of more than four bits (or with 3 and 4 bits on
 *     both sides beyond the K bound) when K >= 16 and M <= 16 (M <= 32 if K <= 8192).
 *   - Otherwise the codes are packed into `workspace` (device, 16-byte aligned, at least
 *     apmm_packed_activation_bytes(M, K, p) bytes, overwritten) and apmm_gemm runs on that: two launches.
 * Without such a workspace the call still takes the one-launch path for every shape of APMM_ALGO_DECODE, and returns
 * APMM_ERR_WORKSPACE (nothing launched) for all others, also those that a workspace of that size would send the same way. */
apmm_status apmm_gemm_from_codes(int64_t M, int64_t N, int64_t K, int p, int q,
                                 const uint8_t *a_codes, const void *w_packed,
                                 int32_t *c_i32, uint16_t *c_f16,
                                 const uint16_t *w_scale, const uint16_t *a_scale,
                                 void *workspace, size_t workspace_bytes, void *stream);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc): apmm_gemm_from_codes without the workspace argument.  The packed activations go into
 * a buffer of APMM_NOALLOC_MAX_PACKED_BYTES bytes that is part of the library's device code (one per GPU, held
 * until the process ends); the call allocates and frees nothing.  Arguments, result and kernel choice as in
 * apmm_gemm_from_codes with a workspace of that size.
 *   - Returns APMM_ERR_WORKSPACE (nothing launched) when apmm_packed_activation_bytes(M, K, p) exceeds
 *     APMM_NOALLOC_MAX_PACKED_BYTES, whether or not the shape would have needed the buffer.
 *   - Every call on one GPU uses that GPU's one buffer, from the packing launch to the end of the GEMM that
 *     follows it on `stream`: calls that overlap on one GPU (different streams, or different threads) race.
 *     Calls on one stream are ordered and safe.  Nothing in the buffer has to be cleared between calls: the
 *     packing writes every byte the GEMM reads. */
#define APMM_NOALLOC_MAX_PACKED_BYTES ((size_t)8 << 20)
apmm_status apmm_gemm_from_codes_noalloc(int64_t M, int64_t N, int64_t K, int p, int q,
                                         const uint8_t *a_codes, const void *w_packed,
                                         int32_t *c_i32, uint16_t *c_f16,
                                         const uint16_t *w_scale, const uint16_t *a_scale, void *stream);

/* One linear of a grouped call: C = A * W^T with the arguments of apmm_gemm. */
typedef struct apmm_problem {
    int64_t M, N, K;
    const void *a_packed;     /* device, packed M x K activations of p bits; ignored when a_codes is given */
    const void *w_packed;     /* device, packed N x K weights of q bits */
    int32_t *c_i32;           /* device, M x N, or NULL */
    uint16_t *c_f16;          /* device, M x N binary16 bit patterns, or NULL */
    const uint16_t *w_scale;  /* device, N, or NULL */
    const uint16_t *a_scale;  /* device, M, or NULL */
    const uint8_t *a_codes;   /* device, M x K unpacked activation codes as for apmm_gemm_from_codes, or NULL */
} apmm_problem;

/* Paper Sec. 5.2 setting (the linears of a decoder layer, each the MatMul of Sec. 3.2): several independent
 * GEMMs of equal p and q with as few launches as possible (for callers whose
 * linears are small enough that the launch, not the data, bounds them: the q/k/v or gate/up
 * projections of one decoder layer at a few tokens share their activations and can go in one launch).
 * `problems` is a HOST array of `count` entries, read before the call returns.  Each entry obeys the
 * rules of apmm_gemm and gives the same result as apmm_gemm on it.  Small-M problems that the same
 * small-M kernel covers are launched eight at a time; all others are launched one by one.  The outputs
 * of different entries must not overlap.  At most 256 entries.  On an argument error nothing is launched.
 * An entry with a_codes takes its activations unpacked, as apmm_gemm_from_codes does in its one-launch
 * form (no packing launch, no packed buffer); such an entry must be a shape of APMM_ALGO_DECODE, else the call
 * returns APMM_ERR_UNSUPPORTED.  Entries with and without a_codes do not share a launch. */
apmm_status apmm_gemm_grouped(int count, const apmm_problem *problems, int p, int q,
                              void *workspace, size_t workspace_bytes, void *stream);

/* ---- A key/value cache held in four bits, and attention over it: what stands between the q/k/v and the output linears of a
 * decoder layer (paper Sec. 5.2 setting).  Keys and values are bipolar-INT codes of four bits (paper Sec. 3.1, Eq. 1), a scale for each token and head.
 *
 * The cache is two buffers of the caller's, in pages of page_size tokens:
 *   codes   pages x kv_heads x 2 x (page_size * head_dim / 2) bytes, 16-byte aligned; of the 2 the first are keys, the second values
 *             keys    token by token, channel c in byte c / 2, in its low four bits where c is even, else in its high ones
 *             values  by eights of tokens; in one, for channels 4 m to 4 m + 3 (m from 0 to head_dim / 4 - 1) eight 16-bit words, one a
 *                     token, channel 4 m + e in bits 4 e to 4 e + 3
 *   scales  pages x kv_heads x 2 x page_size numbers of the type of the tensors, 16-byte aligned
 * A code u with the scale s stands for (2 u - 15) s.  A page may be copied, moved or shared by several sequences; nothing else refers to its place.
 * Scales are not negative and finite, or NaN (see apmm_kv_write); codes are any.
 *
 * A call works on a batch of sequences: */
typedef enum { APMM_F16 = 0, APMM_BF16 = 1 } apmm_dtype;

typedef struct apmm_kv_cache {
    void *codes, *scales;  /* device */
    int64_t pages;
    int page_size;         /* tokens of a page: a power of two from 16 to 1048576 */
    int kv_heads;          /* 1 to 1024 */
    int head_dim;          /* 64 or 128 */
    int dtype;             /* apmm_dtype of scales, keys, values, queries and results */
} apmm_kv_cache;

typedef struct apmm_kv_batch {
    int sequences;              /* 0 to 65536 */
    int64_t tokens;             /* new tokens of all sequences, up to 2^30: rows of the tensors that the call takes */
    const int32_t *lengths;     /* device, sequences: tokens of each sequence, its new ones included; up to 2^30 */
    const int32_t *starts;      /* device, sequences + 1, ascending from 0 to `tokens`: the new tokens of sequence b, its last ones, are rows starts[b]
                                   to starts[b + 1] - 1; or NULL: each sequence has one (tokens == sequences) */
    const int32_t *page_table;  /* device: token t of sequence b is in page page_table[b * table_stride + t / page_size] */
    int64_t table_stride;       /* elements between rows of the table, >= table_width */
    int64_t table_width;        /* pages of a row, 1 to 2^26; tokens beyond table_width * page_size have no place */
} apmm_kv_batch;
/* A call whose launch would have 2^32 work items or more is refused (APMM_ERR_UNSUPPORTED): writing and reading from tokens x kv_heads of about 2^29 on (sequences of
 * one token: 2^26), attention from sequences x kv_heads of 2^24 on where each has a token.
 * Lengths, starts and page numbers are read on the device and cannot be refused; whatever they are, nothing outside of the buffers is
 * read or written.  A token whose position is negative (more new tokens than the length says), beyond the table or in a page outside of 0 to pages - 1 has no place: it is not written,
 * reads as zeros and is seen by no query.
 * Tensors are tokens x heads x head_dim with head_dim contiguous elements and strides in elements, at any address of their type's
 * alignment; rows that all start at multiples of 16 bytes are read and written faster. */

/* Quantises new keys and values as they are written: of each row x of head_dim numbers
 *   s = max |x| / 15, rounded once to its type,  u = (v + 15) / 2, v the odd integer of [-15, 15] nearest to x / s, the upper one on a tie
 * decided as in exact arithmetic, as apmm_quantize_pack_activations does; a scale that rounds to zero has the code of +1 everywhere.  A row with a
 * number that is not finite gets the scale NaN.  Two tokens of a call must not have the same place. */
apmm_status apmm_kv_write(const apmm_kv_cache *cache, const apmm_kv_batch *batch,
                          const void *k, int64_t k_token_stride, int64_t k_head_stride,
                          const void *v, int64_t v_token_stride, int64_t v_head_stride, void *stream);

/* Reads keys and values of the batch's new tokens back (all tokens of a sequence: as many new ones as its length): (2 u - 15) s rounded once to
 * nearest even; what would round past the type's largest number becomes that. */
apmm_status apmm_kv_read(const apmm_kv_cache *cache, const apmm_kv_batch *batch,
                         void *k, int64_t k_token_stride, int64_t k_head_stride,
                         void *v, int64_t v_token_stride, int64_t v_head_stride, void *stream);

/* Attention of the batch's new tokens over the cache.  Query head h belongs to key/value head h / (q_heads / kv_heads).  The query at position p (its
 * sequence's length less its new tokens, plus its place among them) sees key j of its sequence where
 *   j <= p, and where window > 0 also j > p - window or j < sinks
 * and its result is sum_j softmax_j(scale * q . k_j) v_j over these, zeros where there is none.  Statistics and sums are of 32 bits, the weights of the values are
 * rounded to 11 significant bits (where a sequence has few rows of binary16 numbers, 22), the result once; a weight times value scale below 2^-26 of the largest scale that its row sees
 * may count as nothing, and one below 2^-15 of it may be off by as much.  Accuracy holds for value scales from 2^-96 on (bfloat16; below, values lose bits).
 *   scale     > 0 and finite, 1 / sqrt(head_dim) in most models
 *   window    0 (all keys) to 2^30;  sinks  0 to 2^30, without effect where window is 0
 *   workspace device, 16-byte aligned, apmm_kv_attention_workspace_bytes() bytes of the same arguments (0 for most large calls; a call with a window needs no more); calls that may overlap need one each */
size_t apmm_kv_attention_workspace_bytes(const apmm_kv_cache *cache, const apmm_kv_batch *batch, int q_heads);
apmm_status apmm_kv_attention(const apmm_kv_cache *cache, const apmm_kv_batch *batch, int q_heads,
                              const void *q, int64_t q_token_stride, int64_t q_head_stride,
                              void *out, int64_t out_token_stride, int64_t out_head_stride,
                              float scale, int64_t window, int64_t sinks, void *workspace, size_t workspace_bytes, void *stream);

/* ---- Rotary positions: pairs of a row's channels turned by an angle that its position gives.
 * Of head_dim channels the first 2 * pairs are turned: pair i is channels 2 i and 2 i + 1 (interleaved) or i and i + pairs, and with t = position * frequencies[i] its (a, b) becomes
 *   magnitude * (a cos t - b sin t), magnitude * (b cos t + a sin t);
 * the other channels stay as they are.  The angle is a product of 64 bits, so far positions lose nothing, and the sum is that of 64 bits rounded to 32, then to the rows' type (but where more than 20 bits
 * of a pair cancel, and for numbers below 2^-100).  Scaling for long contexts lies in the frequencies and the magnitude. */
typedef struct apmm_rotation {
    const double *frequencies; /* device, pairs: radians a position */
    int64_t pairs;             /* 1 to head_dim / 2 */
    int interleaved;
    float magnitude;           /* > 0 and finite, 1 in most models */
} apmm_rotation;

/* tokens x heads rows of head_dim (1 to 1024) channels; positions: device, one of each token, of any sign.  `inverse`: by -t.  That is also the gradient: of y = apmm_rotary(x) the gradient of x is
 * apmm_rotary, inverse, of y's.  `out` may be x with the same strides, else they must not overlap. */
apmm_status apmm_rotary(int64_t tokens, int heads, int head_dim, int dtype, const void *x, int64_t x_token_stride, int64_t x_head_stride, const int32_t *positions, const apmm_rotation *rotation,
                        int inverse, void *out, int64_t out_token_stride, int64_t out_head_stride, void *stream);

/* apmm_rotary of queries (into q_out, which may be q with the same strides) and of keys, and apmm_kv_write of these keys and of the values, in one launch, with the results of the calls one by one.
 *   q_heads    0 to 2048; 0: no queries, q and q_out may be NULL
 *   q_out      rows that overlap nothing else of the call, or q
 *   positions  device, one of each new token; or NULL: its place in its sequence.  (After apmm_kv_evict places are not positions any more.)
 * Rows of q that belong to no sequence are left as they are in q_out. */
apmm_status apmm_kv_write_rotary(const apmm_kv_cache *cache, const apmm_kv_batch *batch, int q_heads, const int32_t *positions, const apmm_rotation *rotation,
                                 const void *q, int64_t q_token_stride, int64_t q_head_stride, void *q_out, int64_t q_out_token_stride, int64_t q_out_head_stride,
                                 const void *k, int64_t k_token_stride, int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride, void *stream);

/* ---- Keeping the cache within a budget.
 * What attention gives each cached token: for key j of sequence b and key/value head h
 *   weights[b][h][j] = decay * weights[b][h][j] + sum over the sequence's new tokens i and the query heads of h of softmax_j(scale * q_i . k_j)
 * over the keys that apmm_kv_attention with the same arguments lets query i see; a decay of 0 does not read what was there.  weights: device, sequences x kv_heads x capacity 32-bit floats with contiguous
 * tokens; tokens from `capacity` on have none, tokens behind a sequence's length and sequences without new tokens keep what is there.  A query with a score that is NaN (a scale or a number of it is) gives NaN to
 * the keys that it sees.  Results do not depend on the order of execution.
 *   workspace  device, 16-byte aligned, apmm_kv_weights_workspace_bytes() bytes of the same arguments (a call with a window needs no more; about as much as the queries, and up to 256 MiB where
 *              sequences have few); calls that may overlap need one each */
size_t apmm_kv_weights_workspace_bytes(const apmm_kv_cache *cache, const apmm_kv_batch *batch, int q_heads);
apmm_status apmm_kv_weights(const apmm_kv_cache *cache, const apmm_kv_batch *batch, int q_heads, const void *q, int64_t q_token_stride, int64_t q_head_stride,
                            float *weights, int64_t weights_sequence_stride, int64_t weights_head_stride, int64_t capacity, float decay, float scale, int64_t window, int64_t sinks,
                            void *workspace, size_t workspace_bytes, void *stream);

/* Of each sequence and key/value head the first `sinks` tokens, the last `recent` and of the others the heaviest, min(budget, length) in all, copied in their order to places 0, 1, ... of the pages that
 * `to_table` names.  Of equal weights the token of the lower place stays; NaN, and a token from `capacity` on, is lighter than any number.  Tokens without a page never stay.  Heads of a sequence keep
 * equally many tokens, as a rule different ones.
 *   to_table    device, sequences x to_width (rows to_stride apart): pages that no sequence of the call has; a token without a place there is not copied.  The old pages stay as they are.
 *   to_lengths  device, sequences: tokens that stay; not `lengths` itself
 *   kept        device, sequences x kv_heads x budget: the places they had, ascending, then -1
 *   to_weights  device, sequences x kv_heads x budget: their weights (0 for those that have none), then 0; no part of `weights`
 *   workspace   device, 16-byte aligned, apmm_kv_evict_workspace_bytes() bytes of the same sizes (0, then it may be NULL, for tables of up to 65536 tokens); calls that may overlap need one each
 * sinks + recent <= budget.  A call of 2^32 work items or more is refused: sequences x kv_heads from 2^22 on, sequences x kv_heads x budget from about 2^29 on. */
size_t apmm_kv_evict_workspace_bytes(const apmm_kv_cache *cache, int sequences, int64_t table_width);
apmm_status apmm_kv_evict(const apmm_kv_cache *cache, int sequences, const int32_t *lengths, const int32_t *page_table, int64_t table_stride, int64_t table_width,
                          const float *weights, int64_t weights_sequence_stride, int64_t weights_head_stride, int64_t capacity, int64_t budget, int64_t sinks, int64_t recent,
                          const int32_t *to_table, int64_t to_stride, int64_t to_width, int32_t *to_lengths, int32_t *kept, float *to_weights, void *workspace, size_t workspace_bytes, void *stream);

/* ---- Four-bit weights with group scales times activations of 16 bits: y = x * W^T with W[n][k] = (2 u[n][k] - 15) * scales[n][k / group], u bipolar-INT codes of four bits (paper Sec. 3.1, Eq. 1).
 * For layers whose activations are not to be quantised.  The products of a group are exact and summed in 32 bits, its sum is multiplied with the scale in 32 bits, y is rounded once.  (Activations of
 * 2^115 and more may overflow the sums.  Infinities and NaN reach the results of their own row alone.)
 *   group     32, 64 or 128 inputs; the last one of a channel may be shorter
 *   dtype     apmm_dtype of x, y and the scales; the packed form is made for one of them and for its group, and does not tell which
 *   codes     device, N x K uint8, row-major, the low four bits count;  scales  device, N x ceil(K / group)
 *   packed    device, apmm_w4_packed_bytes(N, K, group) bytes, 16-byte aligned, opaque, of this version of the library
 *   x, y      device, M x K and M x N, rows x_stride and y_stride elements apart, at any address of their type's alignment, y's without a part of x; M up to 2^20, N and K up to 2^24
 *   workspace device, 16-byte aligned, apmm_w4_workspace_bytes() bytes of the same sizes (0, then it may be NULL, for many of them); calls that may overlap need one each */
size_t apmm_w4_packed_bytes(int64_t N, int64_t K, int group);
apmm_status apmm_w4_pack(const uint8_t *codes, const void *scales, int64_t N, int64_t K, int group, int dtype, void *packed, void *stream);
size_t apmm_w4_workspace_bytes(int64_t M, int64_t N, int64_t K, int group);
apmm_status apmm_w4_gemm(int64_t M, int64_t N, int64_t K, int group, int dtype, const void *x, int64_t x_stride, const void *packed, void *y, int64_t y_stride,
                         void *workspace, size_t workspace_bytes, void *stream);

/* Measurement aid.  The next apmm_gemm / apmm_gemm_ex / apmm_gemm_from_codes call of the calling thread, if it
 * runs the large-tile MFMA kernel or a small-M kernel in one launch, attaches the two hipEvent_t (created by the
 * caller; either may be NULL) to that kernel's dispatch itself (hipExtLaunchKernel): afterwards they hold the
 * kernel's own begin and end, without the dispatch gaps that events recorded before and after the call include.
 * A call that runs the general XOR/popcount kernel drops them. */
apmm_status apmm_time_next_gemm(void *start_event, void *stop_event);

/* Measurement aid.  Name, with its template arguments, of the GEMM kernel that the last GEMM call of the calling
 * thread launched ("" before the first), e.g. "gemm_mfma_direct_kernel<2,1,4,4,3>" (activation bits, weight bits,
 * wave tile in 32-row and 32-column blocks, store phases).  The string is the calling thread's and stays until it asks again. */
const char *apmm_last_gemm_kernel(void);

const char *apmm_status_string(apmm_status status);
/* Text of the last error on the calling thread ("" if none). */
const char *apmm_last_error(void);
/* Version of the library and of its packed form.  A packed buffer is opaque and carries no mark of its own: one that was
 * written by another version is neither recognised nor refused, and is multiplied wrongly where the form differs, so a program
 * that keeps packed weights in a file keeps this number beside them and packs anew when it has changed.
 * 101: other contents than 100 in packed weights of 3 to 8 bits and packed activations of 5 to 8 bits, sizes as before. */
int apmm_version(void);

#ifdef __cplusplus
}
#endif
#endif /* APMM_H */
