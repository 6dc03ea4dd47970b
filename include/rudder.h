/*
 * rudder.h -- C ABI of the B200 (sm_100a) implementation of the SteerQuant / Rudder inference hot
 * path: the quantized linear layer of a world-action-model diffusion Transformer.
 *
 * One weight matrix per layer is quantised offline to 4 bits with the shared channel scaling D
 * folded in (Eq. 6; Section 4.2, last paragraph) and then serves every token stream and every
 * denoising step.  At run time a first kernel applies D^-1 and the per-stream, per-step gain
 * gamma on the fly while quantising the activations, and writes only the codes Q_X and one row
 * scale r_i (Section 4.4, first kernel; Eq. 8); a second kernel runs the low-bit GEMM and fuses
 * dequantisation, inverse-gain compensation and bias in its epilogue (Section 4.4, Eq. 10).
 *
 * General rules
 *   - Every pointer is a DEVICE pointer unless its comment says HOST.
 *   - The caller owns every buffer it passes (inputs, outputs, workspace).  The library owns only
 *     the memory inside a rudder_weight, allocated by rudder_pack_weights and released by
 *     rudder_weight_free.
 *   - Calls enqueue work on the given CUDA stream (a cudaStream_t passed as void*; NULL = the
 *     default stream) and return without synchronising, except where stated.  rudder_linear,
 *     rudder_block and rudder_quantize_activations allocate nothing.
 *   - Argument errors are detected on the host before anything is launched; nothing traps.
 *   - Device-side waits are bounded: a kernel that gives up records RUDDER_ERR_TIMEOUT in a device
 *     status word that rudder_device_status reads.
 *   - bf16 / fp16 values are passed as their 16-bit patterns (uint16_t).
 *   - Non-finite inputs are undefined behaviour (not checked).
 *   - A rudder_weight belongs to the device that was current when it was packed or imported.  Every call
 *     that takes one must be made with that device current and with buffers of that device; a call made
 *     with another device current returns RUDDER_ERR_ARG before anything is launched.
 *   - Host threads may call concurrently on different streams as long as they share no workspace;
 *     per-device state that is created on first use is guarded inside the library.
 *
 * Shapes: X is [M, K] row-major with leading dimension ldx (elements), W is [N, K] row-major (K
 * contiguous: the transpose of the paper's W in Y = X W), Y is [M, N] with leading dimension ldy.
 * K % 128 == 0, N % 64 == 0, M >= 1.  X, Y 16-byte aligned, ldx % 8 == 0, ldy % 8 == 0.
 */
#ifndef RUDDER_H
#define RUDDER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RUDDER_OK = 0,
    RUDDER_ERR_ARG = 1,          /* NULL required pointer, step outside [0,T), bad segments / stream id */
    RUDDER_ERR_SHAPE = 2,        /* unsupported M / N / K / group */
    RUDDER_ERR_ALIGN = 3,        /* pointer or leading dimension alignment */
    RUDDER_ERR_UNSUPPORTED = 4,  /* scheme / mode combination not available */
    RUDDER_ERR_WORKSPACE = 5,    /* workspace NULL, misaligned or too small */
    RUDDER_ERR_CUDA = 6,         /* a CUDA runtime / driver call failed */
    RUDDER_ERR_TIMEOUT = 7       /* a bounded device-side wait gave up */
} rudder_status;

/* Activation / weight number formats.  Weights are always 4-bit. */
typedef enum {
    RUDDER_W4A8_INT = 0,    /* INT4 weights (group scales), INT8 activations, q_max = 127 (Eq. 1, k = 8) */
    RUDDER_W4A4_INT = 1,    /* INT4 weights, INT4 activations, q_max = 7 (Eq. 1, k = 4); 8-bit tensor-core path
                               (integer MMA, or its exact E4M3 / FP32-accumulator form when group <= 128:
                               same integers, same results) */
    RUDDER_W4A4_NVFP4 = 2   /* E2M1 codes with a UE4M3 scale per 16 elements and an fp32 outer scale */
} rudder_scheme;

/* How the activation range a_i of Eq. 1 (c = a_i) is chosen. */
typedef enum {
    RUDDER_RANGE_PER_TOKEN = 0,  /* a_i = max_k |v_ik| of the scaled row */
    RUDDER_RANGE_STATIC = 1      /* a_i = clip[step]: the paper's calibrated threshold c_tau shared by all streams */
} rudder_range_mode;

typedef struct rudder_weight rudder_weight;   /* opaque; library-owned device memory */

/* Layer-step lookup table of calibrated gains and thresholds (Section 4.3, last paragraph). */
typedef struct {
    const float* gamma;      /* [T, S] gains gamma_{tau,s} > 0 */
    const float* clip;       /* [T] thresholds c_tau > 0, or NULL (required for RUDDER_RANGE_STATIC) */
    int T;                   /* denoising steps */
    int S;                   /* streams, 1..16 */
    rudder_range_mode mode;
} rudder_scale_table;

/* Row -> stream map s(i): contiguous segments of rows. */
typedef struct {
    const int32_t* seg_offsets;  /* HOST [n_seg + 1], ascending, seg_offsets[0] = 0, seg_offsets[n_seg] = M */
    const int32_t* seg_stream;   /* HOST [n_seg], each in [0, S) */
    int n_seg;                   /* 1..64 */
} rudder_segments;

/* ---------------------------------------------------------------------------------------------
 * rudder_pack_weights -- offline fold + quantise + pack (Eq. 6; Section 4.2 last paragraph; Eq. 1
 * with k = 4).  V = W diag(d); integer schemes: per (row j, group g of `group` input channels)
 * Delta_W[j,g] = fp16(max|V| / 7), codes = clip(round(V / Delta_W), -7, 7); NVFP4: tensor scale
 * max|V| / 2688, UE4M3 scale per 16 elements, E2M1 codes.  Also keeps dinv = 1 / d for the
 * run-time prologue.
 *   W [N,K] fp32, d [K] fp32 or NULL (= ones).  group: 64, 128 or K (K = the paper's per-output-
 *   channel scales); ignored for NVFP4.  Allocates the handle (cudaMalloc) and SYNCHRONISES the
 *   stream before returning.  *out is NULL on error.
 */
rudder_status rudder_pack_weights(const float* W, const float* d, int N, int K, rudder_scheme scheme,
                                  int group, void* stream, rudder_weight** out);
rudder_status rudder_weight_free(rudder_weight* w);

/* Shape and storage of a packed weight (HOST outputs; any may be NULL). */
rudder_status rudder_weight_info(const rudder_weight* w, int* N, int* K, int* group, int* scheme,
                                 size_t* device_bytes);

/* Canonical (layout-independent) view of a packed weight, for parity checks and storage:
 *   codes  uint8 [N, K/2]: low nibble = even k; INT4 two's complement, or E2M1 (bit 3 = sign)
 *   scales integer schemes: fp16 bit patterns [N, K/group]; NVFP4: UE4M3 bytes [N, K/16]
 *   dinv   fp32 [K];  tensor_scale fp32 [1] (NVFP4; 1.0 otherwise).  Any output may be NULL. */
rudder_status rudder_weight_export(const rudder_weight* w, uint8_t* codes, void* scales, float* dinv,
                                   float* tensor_scale, void* stream);

/* The inverse of rudder_weight_export: builds a packed weight from its canonical view ("stored as packed
 * integers with corresponding quantization scales", Section 4.2, last paragraph), e.g. from a checkpoint
 * written earlier.  Same layouts as above, all DEVICE pointers; tensor_scale is required for NVFP4 and
 * ignored otherwise; group as in rudder_pack_weights.  The handle behaves exactly like the one
 * rudder_pack_weights returned for the exported weight (same bits out of every kernel).  Allocates and
 * SYNCHRONISES the stream, like rudder_pack_weights. */
rudder_status rudder_weight_import(const uint8_t* codes, const void* scales, const float* dinv, const float* tensor_scale,
                                   int N, int K, rudder_scheme scheme, int group, void* stream, rudder_weight** out);

/* ---------------------------------------------------------------------------------------------
 * rudder_linear -- one quantized linear layer for one denoising step (Section 4.4; Eq. 8; Eq. 10):
 *   v_ik = (x_ik * dinv_k) * gamma[step, s(i)];  codes = clip(round(v * q_max / a_i));
 *   r_i = (a_i / q_max) / gamma;  C^(g) = codes . W-codes per weight group (INT32);
 *   Y_ij = bf16( (sum_g fp32(C^(g)_ij) Delta_W[j,g]) * r_i + b_j )      [group = K: exactly Eq. 10]
 * X bf16 [M, ldx], Y bf16 [M, ldy], bias fp32 [N] or NULL.  workspace holds Q_X and r between the
 * two kernels: at least rudder_linear_workspace_bytes(w, M) bytes, 256-byte aligned.
 */
size_t rudder_linear_workspace_bytes(const rudder_weight* w, int M);
rudder_status rudder_linear(const rudder_weight* w, const uint16_t* X, int64_t ldx, int M,
                            const rudder_segments* seg, int step, const rudder_scale_table* tab,
                            const float* bias, uint16_t* Y, int64_t ldy,
                            void* workspace, size_t workspace_bytes, void* stream);

/* rudder_linear_static -- rudder_linear without a caller-supplied workspace.  (The paper has no
 * counterpart: this is a convenience of this library.)
 * For callers that cannot allocate device memory -- code inside a captured or real-time region where
 * cudaMalloc is off limits, plug-ins that only receive input and output buffers, hosts whose memory
 * pool belongs to another component.  Q_X and r are kept in a fixed array of
 * rudder_linear_static_max_workspace_bytes() = 4 MiB that is part of the library image (every GPU
 * that loads the library holds it until the process exits).  The call allocates nothing.
 *   - Same arguments, results and errors as rudder_linear, minus the workspace.  If
 *     rudder_linear_workspace_bytes(w, M) exceeds the 4 MiB array the call returns
 *     RUDDER_ERR_WORKSPACE and launches nothing.
 *   - The first call on each device looks up the array's device address (with that device current);
 *     make that first call before any stream capture begins.
 *   - All calls on a device share the one array, which keeps the previous call's contents; nothing
 *     in it needs clearing between calls.  Two calls whose kernels may overlap on the GPU (different
 *     streams, or concurrent host threads) race on it: serialise them. */
size_t rudder_linear_static_max_workspace_bytes(void);
rudder_status rudder_linear_static(const rudder_weight* w, const uint16_t* X, int64_t ldx, int M,
                                   const rudder_segments* seg, int step, const rudder_scale_table* tab,
                                   const float* bias, uint16_t* Y, int64_t ldy, void* stream);

/* ---------------------------------------------------------------------------------------------
 * rudder_block -- the four quantized linears of one DiT block for one denoising step, replaying
 * caller-supplied inputs (the paper times DiT replay with captured inputs; attention, norms and
 * GELU stay in BF16 outside this library -- Appendix "Quantization" / "Efficiency").
 * Index 0..3 = QKV (H -> 3H), O (H -> H), MLP up (H -> F), MLP down (F -> H).
 */
typedef struct {
    const rudder_weight* w[4];
    const rudder_scale_table* tab[4];
    const float* bias[4];        /* each [N_l] or NULL */
    const uint16_t* x[4];        /* replay inputs, bf16 [M, ldx[l]]; x[1..3] may be NULL: chained (see below) */
    int64_t ldx[4];
    uint16_t* y[4];              /* outputs, bf16 [M, ldy[l]] */
    int64_t ldy[4];
} rudder_block_args;

/* Chained layers.  x[l] == NULL for l = 1, 2 or 3 makes that layer read the previous layer's output
 * through the minimal BF16 glue, so that the block runs end to end on the device from x[0] alone:
 *   O    (l = 1): the V third of the QKV output, y[0][:, 2 K_1 .. 3 K_1) -- a stand-in for attention, which
 *                 stays outside this library; requires N_0 == 3 K_1;
 *   up   (l = 2): the O output as it is (no norm / residual); requires N_1 == K_2;
 *   down (l = 3): rudder_gelu of the up output, staged at the end of the workspace; requires N_2 == K_3.
 *                 When the down projection's table has a static range (RUDDER_RANGE_STATIC: the paper's calibrated
 *                 threshold, Section 4.3) and an integer scheme, the GELU is applied INSIDE its prologue: with a_i = c_tau
 *                 the requantisation needs no row reduction, so one elementwise pass reads the up output, applies
 *                 the GELU and writes Q_X and r directly; the activated tensor is never stored (same bits either way).
 * A shape that does not chain returns RUDDER_ERR_SHAPE.  rudder_block_workspace_bytes accounts for the
 * staged GELU output (M x K_3 bf16) when x[3] is NULL.  rudder_block_host takes no NULL inputs. */
size_t rudder_block_workspace_bytes(const rudder_block_args* args, int M);
rudder_status rudder_block(const rudder_block_args* args, int M, const rudder_segments* seg, int step,
                           void* workspace, size_t workspace_bytes, void* stream);

/* rudder_block_dit -- the same four linears wired as one DiT block with its BF16 glue (normalisation, GELU and
 * residual additions stay in BF16: Appendix "Quantization"), run end to end on the device from x[0] alone:
 *     h   = x + O( V-third of QKV( rmsnorm(x; norm1_weight) ) )      [the V third stands in for attention, which stays outside]
 *     out = h + down( gelu( up( rmsnorm(h; norm2_weight) ) ) )
 * args->x[0] is the block input [M, H]; args->x[1..3] must be NULL; args->y[l] still receive the four linears' outputs;
 * shapes must be QKV H -> 3H, O H -> H, up H -> F, down F -> H (else RUDDER_ERR_SHAPE).  glue->out [M, ldout] receives
 * the block output.  Workspace: rudder_block_dit_workspace_bytes(args, M), 256-byte aligned.
 * rmsnorm, gelu and the additions are the bit-defined forms of rudder_rmsnorm, rudder_gelu and rudder_add below. */
typedef struct {
    const float* norm1_weight;   /* [H] fp32, 16-byte aligned */
    const float* norm2_weight;   /* [H] fp32, 16-byte aligned */
    float eps;                   /* >= 0 */
    uint16_t* out;               /* bf16 [M, ldout] */
    int64_t ldout;
} rudder_block_glue;
size_t rudder_block_dit_workspace_bytes(const rudder_block_args* args, int M);
rudder_status rudder_block_dit(const rudder_block_args* args, const rudder_block_glue* glue, int M, const rudder_segments* seg,
                               int step, void* workspace, size_t workspace_bytes, void* stream);

/* Measurement hook: rudder_block with a CUDA event between consecutive kernels.  ms (HOST [8])
 * receives the device time of each launch in order: prologue and GEMM of QKV, O, up, down.
 * Creates and destroys its events and SYNCHRONISES the stream before returning. */
rudder_status rudder_block_profile(const rudder_block_args* args, int M, const rudder_segments* seg, int step,
                                   void* workspace, size_t workspace_bytes, void* stream, float* ms);

/* rudder_block for callers whose activations live in HOST memory (pinned for asynchronous copies):
 * args->x[l] and args->y[l] are HOST pointers here (rows contiguous: ldx[l] >= K_l, ldy[l] >= N_l);
 * everything else is as in rudder_block.  Each input is copied to `staging`, the block runs, each
 * output is copied back, without synchronising: work queued on `stream` before the call precedes it,
 * work queued after the call follows the last copy.  Inside, uploads and downloads run on two
 * library-owned streams (created on first use, one pair per device) so that they overlap each other
 * and the kernels; concurrent host threads must therefore not call this on the same device.
 * staging: device memory of at least rudder_block_host_staging_bytes(args, M) bytes, 256-byte
 * aligned. */
size_t rudder_block_host_staging_bytes(const rudder_block_args* args, int M);
rudder_status rudder_block_host(const rudder_block_args* args, int M, const rudder_segments* seg, int step,
                                void* staging, size_t staging_bytes, void* workspace, size_t workspace_bytes,
                                void* stream);

/* ---------------------------------------------------------------------------------------------
 * Parity hooks: the production kernels, with their intermediate results written in canonical form.
 */
/* First kernel alone (Section 4.4): codes int8 [M, K] one code per byte (integer schemes) or
 * uint8 [M, K/2] packed E2M1, low nibble = even k (NVFP4); block_scales UE4M3 [M, K/16] (NVFP4
 * only, else NULL); row_scale fp32 [M]. */
rudder_status rudder_quantize_activations(const rudder_weight* w, const uint16_t* X, int64_t ldx, int M,
                                          const rudder_segments* seg, int step,
                                          const rudder_scale_table* tab, void* codes,
                                          uint8_t* block_scales, float* row_scale, void* stream);
/* The fused pass of a chained down projection alone (see rudder_block): X is the tensor BEFORE the GELU; the codes
 * (int8 [M, K], one per byte) and row scales are those of bf16(gelu(X)).  Static range and integer schemes only
 * (RUDDER_ERR_UNSUPPORTED otherwise). */
rudder_status rudder_gelu_quantize_activations(const rudder_weight* w, const uint16_t* X, int64_t ldx, int M,
                                               const rudder_segments* seg, int step, const rudder_scale_table* tab,
                                               void* codes, float* row_scale, void* stream);
/* rudder_linear that also writes the INT32 group accumulators C^(g) (Section 4.4: "accumulates
 * C = Q_X Q_W in INT32") of rows [row0, row0+rows) x columns [col0, col0+cols) into
 * acc int32 [K/group][rows][cols].  Integer schemes only.  row0 % 128 == 0 and col0 % 64 == 0. */
rudder_status rudder_linear_dump_acc(const rudder_weight* w, const uint16_t* X, int64_t ldx, int M,
                                     const rudder_segments* seg, int step, const rudder_scale_table* tab,
                                     const float* bias, uint16_t* Y, int64_t ldy,
                                     void* workspace, size_t workspace_bytes, void* stream,
                                     int row0, int rows, int col0, int cols, int32_t* acc);

/* BF16 GELU, elementwise, Y = bf16(gelu(X)): the glue of a chained block (the paper keeps GELU in BF16,
 * Appendix "Quantization"; which GELU is not stated).  Reading: the tanh form
 *   gelu(x) = x/2 (1 + tanh(0.7978845608 (x + 0.044715 x^3)))
 * with tanh u replaced by its [7/6] Pade approximant
 *   u (135135 + 17325 u^2 + 378 u^4 + u^6) / (135135 + 62370 u^2 + 3150 u^4 + 28 u^6)   for |u| < 5, +-1 beyond,
 * evaluated in fp32 by Horner's rule from the highest power, every add, multiply and the one divide
 * rounded to nearest on its own (no fused multiply-add): the result is defined bit for bit.
 * X, Y bf16 [M, ld]; N % 8 == 0; 16-byte aligned pointers, leading dimensions multiples of 8. */
rudder_status rudder_gelu(const uint16_t* X, int64_t ldx, int M, int N, uint16_t* Y, int64_t ldy, void* stream);

/* BF16 RMS normalisation of every row with a weight per channel (which normalisation the paper's models use is not
 * stated; reading: RMSNorm): Y = bf16((x * r) * weight), r = 1 / sqrt(mean(x^2) + eps).  Defined bit for bit: fp32, one
 * warp per row, lane l adds x * x (product and sum rounded separately) of the 8-value pieces l, l + 32, ... in order; the
 * 32 partial sums are combined by the exchange l ^ 16, 8, 4, 2, 1; mean = sum / N, r by IEEE division and square root.
 * X, Y bf16 [M, ld], weight fp32 [N]; N % 8 == 0; 16-byte aligned pointers, leading dimensions multiples of 8. */
rudder_status rudder_rmsnorm(const uint16_t* X, int64_t ldx, int M, int N, const float* weight, float eps, uint16_t* Y, int64_t ldy,
                             void* stream);
/* BF16 residual addition, elementwise: Y = bf16(A + B), one fp32 addition.  Same shape and alignment rules. */
rudder_status rudder_add(const uint16_t* A, int64_t lda, const uint16_t* B, int64_t ldb, int M, int N, uint16_t* Y, int64_t ldy,
                         void* stream);

/* ---------------------------------------------------------------------------------------------
 * Attention over a paged key-value cache, and what stands around it.  (The paper keeps attention, position rotation and the
 * key-value cache in BF16 outside the quantized path -- Appendix "Quantization"; these are this library's own forms of them for
 * the steps of a few action / proprioceptive tokens next to a cached context.)
 *
 * Data that only the device sees (lengths, page ids, slots, positions) is checked by the kernels: a bad value is
 * skipped, never used as an index, and recorded for rudder_device_status as RUDDER_ERR_ARG with `where` = 911 page id,
 * 912 length or row range, 913 position, 914 slot, 915 pages or table columns exhausted, 916 slot map full.
 */
typedef enum {
    RUDDER_CACHE_BF16 = 0,
    RUDDER_CACHE_E4M3 = 1        /* value = code x scale of the head */
} rudder_cache_format;

/* Keys and values of all requests: n_pages pages of page_size tokens (a power of two, 1..1024), `heads` key-value heads of head_dim
 * channels (64, 128 or 256), channels contiguous.  The three strides (elements, multiples of 16 bytes, the same for k and v)
 * put pages, heads and tokens in any order; offsets are 64-bit.  Slot of a token = page id x page_size + place in the page. */
typedef struct {
    void* k;                     /* 16-byte aligned */
    void* v;
    rudder_cache_format format;
    int n_pages, page_size, heads, head_dim;
    int64_t page_stride, head_stride, token_stride;
    const float* k_scale;        /* [heads] fp32 > 0, E4M3 only; NULL = ones */
    const float* v_scale;
} rudder_paged_cache;

/* rudder_page_tables -- page tables and slot maps on the device from the requests' lengths, one launch.
 * Request b holds old_lens[b] tokens and gets new_lens[b] more; pages(l) = ceil(l / page_size).  Requests take pages from
 * free_pages in order:  need_b = pages(old + new) - pages(old),  first_b = sum_{i<b} need_i,
 *     page_table[b][pages(old_b) + j] = free_pages[first_b + j]            for j < need_b
 * starts[b] = sum_{i<b} new_i (starts[B] = all new tokens); token starts[b] + i has position old_b + i and its slot; the
 * capacity - starts[B] rows behind the last token get position and slot -1.  used = sum need_b (above n_free: exhausted -- the
 * tokens without a page get slot -1).  Other table entries are left as they were; calling again with the same inputs writes the same. */
typedef struct {
    const int32_t* old_lens;     /* [B] >= 0 */
    const int32_t* new_lens;     /* [B] >= 0 */
    int B;                       /* 1..8192 */
    int page_size;
    const int32_t* free_pages;   /* [n_free]; may be NULL when n_free is 0 */
    int n_free;
    int32_t* page_table;         /* [B, ld_table], in and out */
    int64_t ld_table;
    int max_pages;               /* columns, <= ld_table */
    int64_t* slots;              /* [capacity] out */
    int32_t* positions;          /* [capacity] out */
    int capacity;                /* 1..2^30 - 1 */
    int32_t* starts;             /* [B + 1] out */
    int32_t* used;               /* [1] out */
} rudder_page_table_args;
rudder_status rudder_page_tables(const rudder_page_table_args* args, void* stream);

/* rudder_qk_norm_rope -- RMS norm of every query and key head, rotation by the row's position, keys and values appended to the
 * cache: one pass over the QKV linear's output.  Per head of D channels: y = (x r) w, r = 1 / sqrt(mean(x^2) + eps); of
 * its first `rot` channels the pairs (i, i + rot/2) (RUDDER_ROPE_HALF) or (2i, 2i + 1) (RUDDER_ROPE_PAIRS) become
 * (y_i c - y_j s, y_j c + y_i s), c and s the entry i of row positions[m] of the tables.  Q = bf16 of the result; K likewise, or in
 * the cache at slots[m] (bf16, or E4M3 of value x (1 / scale), saturating); V = the values unchanged, cache only.
 * Bit-defined: fp32, every operation rounded once.  Sum of squares: D / 8 lanes of 8 channels -- lane l < rot / 8 the channels 4l .. 4l + 3
 * and the same + rot/2 with RUDDER_ROPE_HALF, else 8 neighbours -- each its even places in order, its odd places in order, then
 * the two; the lanes combined by the exchange l ^ D/16, .., 1.
 * A row with positions[m] < 0 is padding and left as it was; one with slots[m] < 0 is not appended.  Slots of one call are
 * distinct (which of two equal ones stays is not defined).  Q may be X itself (same leading dimension) and K the keys' place in X. */
typedef enum { RUDDER_ROPE_HALF = 0, RUDDER_ROPE_PAIRS = 1 } rudder_rope_style;
typedef struct {
    const uint16_t* X;           /* bf16 [M, ldx]: heads x D query, kv_heads x D key, kv_heads x D value channels */
    int64_t ldx;
    int M;
    int heads, kv_heads, head_dim;   /* head_dim 64, 128 or 256; heads up to 1024 */
    const float* q_weight;       /* [D] fp32, 16-byte aligned, or NULL = ones */
    const float* k_weight;
    float eps;                   /* >= 0 */
    const float* cos;            /* fp32 [n_pos, rot / 2]; not read when rot is 0 */
    const float* sin;
    int n_pos, rot;              /* rot a multiple of 16, 0..D */
    rudder_rope_style style;
    const int32_t* positions;    /* [M]; may be NULL when rot is 0 */
    uint16_t* Q;                 /* bf16 [M, ldq] */
    int64_t ldq;
    uint16_t* K;                 /* bf16 [M, ldk], or NULL with cache and slots */
    int64_t ldk;
    const rudder_paged_cache* cache;
    const int64_t* slots;        /* [M] */
} rudder_qk_args;
rudder_status rudder_qk_norm_rope(const rudder_qk_args* args, void* stream);

/* rudder_attention_paged -- attention of the new tokens of each request over its cached keys and values:
 *     s_j = scale q . k_j,  O = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  lse = m + ln sum_j exp(s_j - m)
 * over j < kv_lens[b] (the new tokens' own keys included when they have been appended); with `causal` token t of n sees
 * j <= kv_lens[b] - n + t.  Query head h uses key-value head h / (heads / cache heads).  A row that sees no key gets zeros and
 * lse = -infinity.  What the cache holds at and behind kv_lens[b] is never used, and what a row does not see has no part in it (not a
 * number or infinite as it may be).  A value that a row sees and that is infinite or not a number makes that channel of the row infinite or not a number.
 * Rounding: scores and sums fp32; probabilities to 2^-17 with a bf16 cache; with E4M3 to 2^-11, those below 2^-25 of a row's largest to 2^-36 of that.
 * Request b has the rows q_starts[b] .. q_starts[b+1] - 1 (at most max_q), or with q_starts NULL the rows b max_q ..
 * (b + 1) max_q - 1; all other rows of O and lse are left as they were.  O may be Q.
 * workspace: rudder_attention_workspace_bytes(args) bytes (from heads, max_q and the cache's shape alone), 256-byte
 * aligned, contents irrelevant; calls that may overlap on the GPU need one each.  Results do not depend on timing. */
typedef struct {
    const uint16_t* Q;           /* bf16 [M, ldq], heads x D */
    int64_t ldq;
    int M;
    int heads;                   /* a multiple of cache->heads */
    const rudder_paged_cache* cache;
    const int32_t* page_table;   /* [B, ld_table] */
    int64_t ld_table;
    int max_pages;               /* columns that may be read; max_pages x page_size <= 2^31 - 2^16 */
    const int32_t* kv_lens;      /* [B] */
    const int32_t* q_starts;     /* [B + 1] or NULL */
    int B, max_q;
    int causal;
    float scale;
    uint16_t* O;                 /* bf16 [M, ldo] */
    int64_t ldo;
    float* lse;                  /* fp32 [M, heads] or NULL */
} rudder_attention_args;
size_t rudder_attention_workspace_bytes(const rudder_attention_args* args);
rudder_status rudder_attention_paged(const rudder_attention_args* args, void* workspace, size_t workspace_bytes, void* stream);

/* rudder_linear_a16 -- 1 to 16 rows through a packed weight with the activations kept in 16 bits (a step embedding, a
 * handful of action tokens): Y_mj = bf16( sum_k (x_mk dinv_k) q_jk Delta_W[j, g(k)] + b_j ), no workspace, any scheme.
 * The gains of Eq. 8 cancel without an activation quantiser, so there are no segments, steps or tables.  fp32 sums; x dinv
 * enters the product with 16 significant bits (from halfway between the largest bf16 number and 2^128 on: as infinity).  K up to 36864 (one launch; wide layers one per pass of
 * rows: above K = 9216 8 at a time, above 17920 4).  Other shape and alignment rules as in rudder_linear. */
rudder_status rudder_linear_a16(const rudder_weight* w, const uint16_t* X, int64_t ldx, int M, const float* bias, uint16_t* Y, int64_t ldy,
                                void* stream);

/* rudder_block_cached -- rudder_block_dit with attention over a paged cache in the place of its stand-in:
 *     h   = x + O( attention( norm and rotation( QKV( rmsnorm(x; norm1_weight) ) ), cache ) )
 *     out = h + down( gelu( up( rmsnorm(h; norm2_weight) ) ) )
 * The M rows are the new tokens of attn->B requests; their keys and values are appended to the cache before attention reads it.
 * Shapes: QKV H -> (heads + 2 kv heads) D, O heads D -> H, up H -> F, down F -> H.  Of `qk` the members X, ldx, M, Q, ldq, K, ldk and of `attn`
 * Q, ldq, M, O, ldo are supplied by the block; both name the same cache.  attn->lse [M, heads] or NULL.  A row of padding (position < 0)
 * attends to nothing, inside a request's rows or outside: its attention output is zero, its lse -infinity (outside: left as it was).  With `causal` it counts
 * as one of its request's rows, so the padding of a request stands in front of its tokens.  Workspace: rudder_block_cached_workspace_bytes(args, attn, M), 256-byte aligned. */
size_t rudder_block_cached_workspace_bytes(const rudder_block_args* args, const rudder_attention_args* attn, int M);
rudder_status rudder_block_cached(const rudder_block_args* args, const rudder_block_glue* glue, const rudder_qk_args* qk,
                                  const rudder_attention_args* attn, int M, const rudder_segments* seg, int step, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* Reads and clears the device status word (SYNCHRONISES the device).  *last (HOST) receives
 * RUDDER_OK, RUDDER_ERR_TIMEOUT or RUDDER_ERR_ARG (bad device data, see above); *where (HOST, may be NULL) a code
 * naming the wait that gave up or what was bad. */
rudder_status rudder_device_status(int* last, int* where);

/* Self-test of the bounded-wait path (no counterpart in the paper): launches ONE warp that waits, for at
 * most limit_cycles SM clocks (1e3 .. 1e8), on a barrier that nothing signals -- no copy, no tensor memory,
 * nothing in flight -- gives up, records RUDDER_ERR_TIMEOUT with the wait code 901 in the device status word
 * and returns normally.  The context stays usable; rudder_device_status then reports and clears the word. */
rudder_status rudder_selftest_wait_timeout(long long limit_cycles, void* stream);

const char* rudder_status_string(rudder_status s);

#ifdef __cplusplus
}
#endif
#endif /* RUDDER_H */
