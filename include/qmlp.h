/*
 * qmlp.h -- C ABI of the MI355X (gfx950) W4/W2-GateUp decode-MLP library.
 *
 * The library runs the inference hot path of the W4/W2-GateUp deployment
 * with Recover-LoRA adapters (arXiv 2606.04238): one gated-MLP block whose
 * gate and up projections are 2-bit group-quantized, each carrying an
 * unmerged low-rank correction x A^T B^T, followed by SiLU(gate) * up and a
 * 4-bit group-quantized down projection.
 *
 *   Sec. 3.1, Eq. (1)  LoRA-augmented linear  Y = W X + alpha B A X.
 *   Sec. 3.3           W4/W2-GateUp: gate/up at 2 bits, every other linear
 *                      (down included) at 4 bits, group-wise quantization.
 *   Sec. 4.1           Stage 1: gate/up to INT2 by post-training quantization.
 *   Sec. 4.2           adapters on the quantized gate/up, kept as a separate
 *                      module at inference (not merged into the 2-bit grid).
 *   Sec. 5             the MLP is one fused gate-activation-down operator;
 *                      decode is bound by the bandwidth of loading weights.
 *   Sec. 7             deployment: quantize gate/up to INT2 (step 1), the rest
 *                      to INT4 (step 4), deploy with attached adapters (step 5).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Every pointer except the qmlp_qweight/qmlp_mlp descriptors and the
 *    status-string result is a DEVICE pointer into memory the caller owns.
 *    The library never allocates or frees device memory and keeps no pointer
 *    after a call returns.
 *  - Work is enqueued on `stream` (a hipStream_t; NULL = the null stream)
 *    and runs asynchronously; nothing synchronizes.
 *  - Arguments are validated first.  On any error nothing is enqueued and no
 *    output is written.  A HIP launch error maps to QMLP_ERR_HIP; a fault
 *    inside a kernel surfaces at the caller's next synchronization.
 *  - Calls are reentrant: there is no global mutable state.  Inputs and
 *    outputs of one call must not overlap.
 *
 * Storage format of a quantized matrix W [n][k] (nn.Linear orientation:
 * n outputs, k inputs; groups of g consecutive inputs of one row):
 *  - codes: row-major, each row a run of little-endian 32-bit words; code i
 *    of a row sits at bits [b*(i mod 32/b), +b) of word i/(32/b) of that row
 *    (16 codes per word at b=2, 8 at b=4).  Size n*k*b/8 bytes.
 *    At b=3 (Appendix B) a row is two planes: the low two bits of every code
 *    in the 2-bit layout (k/16 words), then the high bit of every code, code
 *    i at bit (i mod 32) of word i/32 of that plane (k/32 words); k % 128 == 0
 *    (rows of 3k/8 bytes stay 16-byte aligned).
 *  - meta: row-major [n][k/g] pairs of binary16 (scale, zero), scale first.
 *    Size n*(k/g)*4 bytes.  The dequantized weight is scale * (q - zero).
 *  - Quantizer (round-to-nearest, asymmetric min-max; the paper fixes only
 *    the bit width and grouping): per group lo = min(0, min w),
 *    hi = max(0, max w), s = (hi - lo)/(2^b - 1) in fp64, scale = s rounded
 *    once to binary16 (nearest-even; 0 becomes 1.0),
 *    zero = clamp(rint(-lo/scale), 0, 2^b - 1) (an integer),
 *    q = clamp(rint(w/scale) + zero, 0, 2^b - 1); rint is nearest-even and
 *    every quotient an IEEE fp64 division.
 *
 * Activation types: x, h, y and the LoRA factors are binary16 (QMLP_F16) on
 * the decode path (1 <= M <= 16) and bfloat16 (QMLP_BF16) on the
 * prefill-chunk path (M a multiple of 128); accumulation is fp32.
 */
#ifndef QMLP_H
#define QMLP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    QMLP_OK = 0,
    QMLP_ERR_NULL = 1,          /* a required pointer is NULL */
    QMLP_ERR_SHAPE = 2,         /* sizes inconsistent or not a supported multiple */
    QMLP_ERR_ALIGN = 3,         /* a device pointer is not 16-byte aligned */
    QMLP_ERR_UNSUPPORTED = 4,   /* bits / group / rank / M / dtype combination not built */
    QMLP_ERR_WORKSPACE = 5,     /* workspace NULL or smaller than qmlp_workspace_bytes() */
    QMLP_ERR_HIP = 6            /* a HIP runtime call failed (launch, attribute, device query) */
} qmlp_status;

typedef enum { QMLP_F16 = 0, QMLP_BF16 = 1 } qmlp_dtype;

/* A hipStream_t passed as an opaque pointer (NULL = the null stream). */
typedef void *qmlp_stream;

/* Non-owning view of one packed quantized matrix in device memory. */
typedef struct {
    int32_t bits;     /* 2 (gate/up) or 4 (down); 3 for gate/up; see qmlp_mlp */
    int32_t n_out;    /* rows n of the logical W [n][k] */
    int32_t k_in;     /* columns k; groups run along k */
    int32_t group;    /* g: 32, 64 or 128; k_in % g == 0 */
    void *codes;      /* qmlp_codes_bytes(bits, n_out, k_in) bytes, 16-B aligned */
    void *meta;       /* qmlp_meta_bytes(n_out, k_in, group) bytes, 16-B aligned */
} qmlp_qweight;

/* One W4/W2-GateUp MLP block with its Recover-LoRA adapters (Sec. 3.3, 4.2).
 * gate/up at 2 bits and down at 4 bits, groups of 64 or 128, is the block
 * every path takes.  The binary16 decode path (qmlp_forward,
 * qmlp_forward_layers, qmlp_forward_batch; not the one-kernel layer, the
 * streamed and matrix-core launches nor the persistent stack, which take
 * only that form) also runs the comparison
 * points of the throughput analysis (Sec. 5.2) and the paper's INT2 grouping
 * (Sec. 3.3, Sec. 4.1): gate/up at 4 bits (uniform W4), down at 2 bits
 * (uniform W2, groups of 64 or 128), and group 32 for gate/up (any width)
 * and for a 4-bit down; and the 3-bit gate/up of Appendix B (W3, group 32
 * in the paper; 64 and 128 also accepted). */
typedef struct {
    qmlp_qweight gate;      /* bits 2 (or 3, 4), [f][d] */
    qmlp_qweight up;        /* same bits and group as gate, [f][d] */
    qmlp_qweight down;      /* bits 4 (or 2), [d][f] */
    const void *A_gate;     /* [rank][d] activation type (nn.Linear / PEFT "lora_A") */
    const void *B_gate;     /* [f][rank] activation type (PEFT "lora_B")            */
    const void *A_up;       /* [rank][d] */
    const void *B_up;       /* [f][rank] */
    int32_t rank;           /* r: 0 (no adapter), 8, 16 or 32 */
    float lora_scale;       /* multiplies B A x (Eq. (1)'s alpha; PEFT: alpha/r) */
} qmlp_mlp;

/* ---------------------------------------------------------------- sizes */

/* Bytes of packed codes for an [n_out][k_in] matrix at `bits` (0 if invalid). */
size_t qmlp_codes_bytes(int bits, int n_out, int k_in);

/* Bytes of (scale, zero) metadata for [n_out][k_in] at group `group` (0 if invalid). */
size_t qmlp_meta_bytes(int n_out, int k_in, int group);

/* Workspace bytes qmlp_forward / qmlp_gateup_w2_lora need for this block at
 * M tokens (0 if the combination is unsupported).  Layout: a 1024-byte
 * control block (uint32 words, each on its own 128-byte line: word 0 counts
 * the one-kernel layer's calls, word 32 its finished blocks, word 160 holds
 * sticky error bits: 1 = t wait timed out, 2 = h wait timed out), then t
 * (fp32), h (activation type [M][f]), on the prefill path lora_scale * t in
 * bfloat16, and on the decode path the one-kernel layer's tagged hand-off
 * words (one [4][64] block of 64-bit words per compute unit, [4][f] 32-bit;
 * where the block's launches on the matrix cores need more bytes than those,
 * for LoRA-A's slices and the fp32 partial sums [slices][M][d] of long down
 * rows, as many as they need), and on the prefill path, when the down projection splits f into slices
 * to fill the chip, the slices' fp32 partial sums [S][M][d].  The calls
 * also take a decode workspace without the bytes for long down rows beyond
 * the hand-off words; they then run the stand-alone kernel, which is slower.
 * The workspace must be ZERO before
 * its first call, and zeroed again before it serves a block of another shape
 * or after an error bit appeared (the results of that call are invalid).
 * One workspace serves one call at a time: calls that overlap in time on the
 * same workspace race. */
size_t qmlp_workspace_bytes(const qmlp_mlp *mlp, int M, qmlp_dtype dtype);

/* ----------------------------------------------------- packing (offline) */

/*
 * Sec. 4.1 / Sec. 7 step 1: quantize fp32 W [n_out][k_in] (row-major,
 * device) to 2-bit codes, group `group` along k_in, writing out->codes and
 * out->meta (caller-allocated, sizes from qmlp_codes_bytes/qmlp_meta_bytes).
 * On success out->bits/n_out/k_in/group are filled in.
 * A group holding a non-finite weight or whose scale overflows binary16 is
 * written as codes 0, scale NaN (0x7E00), zero 0, and bit 0 of *d_status
 * (a device int32, may be NULL) is set with an atomic OR; the caller zeroes
 * *d_status beforehand.  Requires group in {32, 64, 128}, k_in % group == 0
 * (32 is the paper's INT2 group).
 */
qmlp_status qmlp_pack_w2(const float *W, int n_out, int k_in, int group,
                         qmlp_qweight *out, int32_t *d_status, qmlp_stream stream);

/* Appendix B: the same at 3 bits (the W3 gate/up variant), in the two-plane
 * layout above.  Requires group in {32, 64, 128}, k_in % 128 == 0. */
qmlp_status qmlp_pack_w3(const float *W, int n_out, int k_in, int group,
                         qmlp_qweight *out, int32_t *d_status, qmlp_stream stream);

/* Sec. 3.3 / Sec. 7 step 4: the same at 4 bits (down projection and every
 * other non-gate/up linear).  Requires group in {32, 64, 128}, k_in % group == 0. */
qmlp_status qmlp_pack_w4(const float *W, int n_out, int k_in, int group,
                         qmlp_qweight *out, int32_t *d_status, qmlp_stream stream);

/* ------------------------------------------------------ the hot path */

/*
 * Sec. 3.1 Eq. (1) on the gate and up projections, then the activation of
 * the fused gate-activation-down operator (Sec. 5):
 *   G = W2gate x + lora_scale * B_gate (A_gate x)
 *   U = W2up   x + lora_scale * B_up   (A_up   x)
 *   h = SiLU(G) * U = G / (1 + exp(-G)) * U
 * x [M][d] and h [M][f] are row-major in the activation type `dtype`.
 * ws/ws_bytes: workspace of at least qmlp_workspace_bytes(mlp, M, dtype).
 * M == 0 enqueues nothing and returns QMLP_OK.  Gate and up must be 2-bit
 * (group 32 allowed on the decode path); QMLP_ERR_UNSUPPORTED otherwise.
 */
qmlp_status qmlp_gateup_w2_lora(const qmlp_mlp *mlp, const void *x, int M, qmlp_dtype dtype,
                                void *h, void *ws, size_t ws_bytes, qmlp_stream stream);

/*
 * The 4-bit down projection (Sec. 3.3): y [M][n_out] = W4down h, with
 * h [M][k_in] and y row-major in the activation type.  No workspace (longer
 * rows than those named at qmlp_linear_batch run the stand-alone kernel).
 * Group 32 only on the binary16 decode path.
 */
qmlp_status qmlp_down_w4(const qmlp_qweight *down, const void *h, int M, qmlp_dtype dtype,
                         void *y, qmlp_stream stream);

/*
 * The whole block, y = W4down(SiLU(G) * U) (Sec. 3.3, 4.2, 5), x [M][d] ->
 * y [M][d].  The intermediate h lives only in the workspace.
 */
qmlp_status qmlp_forward(const qmlp_mlp *mlp, const void *x, int M, qmlp_dtype dtype,
                         void *y, void *ws, size_t ws_bytes, qmlp_stream stream);

/*
 * qmlp_forward without a workspace argument, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  The block's workspace is a fixed array
 * of qmlp_noalloc_scratch_bytes() (1 MiB) in this library's device memory,
 * one per GPU, held until the process ends; the call allocates and frees
 * nothing.  Binary16 decode only (1 <= M <= 16): QMLP_ERR_UNSUPPORTED for
 * bfloat16, QMLP_ERR_WORKSPACE when the smallest workspace qmlp_forward
 * takes exceeds the array (on 256 compute units the Qwen3-4B block fits up to
 * M = 16, the Qwen3-8B one up to M = 13, the 14B-class one up to M = 7; d =
 * 8192, f = 32768 does not).  Each call first clears the part of the array
 * the block uses (one small fill kernel, then the kernels of qmlp_forward,
 * on `stream`), so it never depends on an earlier call's contents.  All
 * calls on one GPU share its array: calls that overlap in time on the same
 * GPU (other streams, other host threads) race.  Other errors as for
 * qmlp_forward; on any error nothing is enqueued.
 */
qmlp_status qmlp_forward_noalloc(const qmlp_mlp *mlp, const void *x, int M, qmlp_dtype dtype,
                                 void *y, qmlp_stream stream);

/* Size of the per-GPU array behind qmlp_forward_noalloc.  Host-only. */
size_t qmlp_noalloc_scratch_bytes(void);

/*
 * A stack of L blocks of one shape on a residual stream, as the MLP
 * sub-blocks of an L-layer decoder with the attention sub-blocks left out
 * (Sec. 3.3: each layer carries one gated MLP):
 *   x_0 = x,  u_l = RMSNorm(x_l),  y_l = block_l(u_l),  x_{l+1} = x_l + y_l,
 * RMSNorm(v) = v / sqrt(mean(v^2) + 1e-6) per token with unit gain (a
 * learned gain folds into the input columns of gate, up and LoRA-A before
 * quantization).  u_l and y_l are rounded to binary16, the sum of two
 * binary16 values is rounded once (nearest-even).  Binary16 only.
 * layers[0..L-1] are host descriptors (same d, f, group and rank); x [M][d];
 * y [L][M][d] receives every block's output (layer l at y + l*M*d); x_out
 * [M][d] (may be NULL) receives x_L.  Each y_l equals qmlp_forward of layer
 * l on RMSNorm(x_l) within the output bar.
 *
 * At M = 1 for shapes with f % 256 == 0, d % 512 == 0, d <= 4096,
 * (d/g) % 4 == 0 on a GPU with 8 XCDs of 32 compute units, the stack runs
 * as ONE persistent launch per 40 layers: the weights of block l+1 stream in
 * while block l finishes (weights do not depend on activations), and no
 * step of block l+1 starts before x_{l+1} is complete.  Every other shape
 * runs per block: a norm kernel, qmlp_forward, a residual-add kernel.
 *
 * ws/ws_bytes: at least qmlp_stack_workspace_bytes(layers, L, M, dtype),
 * zero before the first call, with the rules of qmlp_workspace_bytes (after
 * the per-block workspace come three activation buffers, then the
 * persistent launch's 1024-byte control block -- word 0 its step counter,
 * word 64 sticky error bits: 1/2/4 = a wait for the activation / h / the
 * cross-XCD partials gave up, 8 = a workgroup found no place -- and its
 * hand-off words).  Errors as for qmlp_forward; QMLP_ERR_UNSUPPORTED for
 * bfloat16.
 */
size_t qmlp_stack_workspace_bytes(const qmlp_mlp *layers, int L, int M, qmlp_dtype dtype);

qmlp_status qmlp_forward_stack(const qmlp_mlp *layers, int L, const void *x, int M,
                               qmlp_dtype dtype, void *y, void *x_out, void *ws, size_t ws_bytes,
                               qmlp_stream stream);

/* Byte offset, within a qmlp_forward_stack workspace, of the persistent
 * launch's sticky error word (a uint32: 1/2/4 = a wait for the activation /
 * h / the cross-XCD partials gave up, 8 = a workgroup had no place; the
 * word is cleared by the caller when it zeroes the workspace and never by
 * the library); 0 if these blocks do not run persistently or the call would
 * be rejected.  Host-only. */
size_t qmlp_stack_error_offset(const qmlp_mlp *layers, int L, int M, qmlp_dtype dtype);

/* Launches qmlp_forward_stack makes: the number of persistent launches when
 * the stack runs persistently, else the per-layer kernels plus the norm and
 * residual-add kernels; 0 if the call would be rejected.  Host-only. */
int qmlp_stack_launches(const qmlp_mlp *layers, int L, int M, qmlp_dtype dtype);

/*
 * L independent blocks of one shape (Sec. 3.3, 4.2, 5: the gated MLP of each
 * layer of the modelled decoders, with separately seeded weights and
 * inputs): y_l = block_l(x_l) for l = 0..L-1, each exactly the operation of
 * qmlp_forward.  layers[0..L-1] are host descriptors (same d, f, group and
 * rank); x [L][M][d] and y [L][M][d] are row-major in the activation type
 * (block l at x + l*M*d, y + l*M*d).
 *
 * Binary16 blocks run in batches of up to 40.  At M = 1 in the
 * W4/W2-GateUp form (2-bit gate/up, 4-bit down, groups 64/128, rank 0, 8,
 * 16 or 32) with d % 512 == 0, d <= 4096, f % 128 == 0, f <= 12288, a batch
 * STREAMS: one persistent gate/up launch that also computes the LoRA-A
 * products and one persistent down launch, each workgroup owning a
 * contiguous range of the batch's rows flattened over blocks; h of every
 * block passes through the workspace between the two launches.  Every other
 * binary16 batch of two tokens or more (a few short rows at two tokens aside)
 * runs each half that fits on the MATRIX CORES: gate/up at 2 bits with d <= 6144 or at 4 bits with d <= 3072, and any
 * down (one of several slices of f, below, only beside such a gate/up).  The
 * LoRA-A launch (fp32 partial sums over four slices of d, added in slice order
 * by the next launch) is followed by one gate/up launch and one down launch
 * that multiply every unpacked weight into all M tokens with
 * v_mfma_f32_16x16x32_f16; large batches of long rows do so at one token too,
 * and W4/W2-GateUp blocks of longer gate/up rows at 3 to 8 tokens on kernels
 * that keep the activations in LDS.  A half that does not fit (3-bit gate/up,
 * 4-bit gate/up past 3072) and the rest run the stand-alone kernels as
 * qmlp_forward_batch does; bfloat16 runs qmlp_forward once per block.
 *
 * ws/ws_bytes: at least qmlp_layers_workspace_bytes(layers, L, M, dtype)
 * (binary16: that of qmlp_forward_batch, with four times its t area on the
 * matrix cores and twice on the streamed path, and on the matrix cores, where
 * rows of down are longer than one workgroup holds -- f > 6144, f > 12288 at
 * up to eight tokens, half of each at 4 bits in groups of 32 -- fp32 partial
 * sums [slices][min(L,40)][M][d] and 1 KB of counters).  On the streamed path with
 * adapters the gate/up launch also computes LoRA-A and hands t over as
 * tagged words: the control block's word 0 counts the calls and word 160
 * holds sticky error bits (1 = a wait for t gave up), so the workspace must
 * be ZERO before its first call and zeroed again before it serves other
 * blocks' shape or after an error bit; one call at a time per workspace.
 * The other paths keep no state between calls.
 * Errors as for qmlp_forward.
 */
size_t qmlp_layers_workspace_bytes(const qmlp_mlp *layers, int L, int M, qmlp_dtype dtype);

qmlp_status qmlp_forward_layers(const qmlp_mlp *layers, int L, const void *x, int M,
                                qmlp_dtype dtype, void *y, void *ws, size_t ws_bytes,
                                qmlp_stream stream);

/* Which path qmlp_forward_layers takes for these blocks: 1 = streamed, 2 =
 * batched (each half on the matrix cores or the stand-alone kernels), 3 =
 * qmlp_forward per block (bfloat16), 4 = matrix cores (3 <= M <= 16 in the
 * W4/W2-GateUp form, d % 512 == 0, f % 256 == 0); 0 if the call would be
 * rejected.  Host-only (it queries
 * the current device's compute-unit count). */
int qmlp_layers_path(const qmlp_mlp *layers, int L, int M, qmlp_dtype dtype);

/* Launches qmlp_forward_layers makes: per batch of up to 40 blocks 2 on the
 * streamed path, 3 on the matrix-core and batched paths (2 without
 * adapters), or the per-block launches of qmlp_forward; 0 if the call would
 * be rejected.  Host-only. */
int qmlp_layers_launches(const qmlp_mlp *layers, int L, int M, qmlp_dtype dtype);

/*
 * The same L independent blocks as qmlp_forward_layers, always on the
 * stand-alone decode kernels, in batches of up to 40 blocks: the LoRA-A
 * products of every block of a batch (one launch, skipped at rank 0), then
 * gate/up with SiLU(G) * U of every block (one launch), then down of every
 * block (one launch).  Binary16 only (1 <= M <= 16), any width combination
 * qmlp_mlp lists: it is the path of the width comparison (Sec. 5.2), where
 * every precision must run on the same kernels, and of callers that do not
 * want a launch holding every compute unit.  h and t of a batch stay in the
 * workspace between the launches.
 *
 * ws/ws_bytes: at least qmlp_batch_workspace_bytes(layers, L, M, dtype):
 * a 1024-byte block left at zero, t [min(L,40)][M][2r] fp32, h
 * [min(L,40)][M][f] binary16.  No state is kept between calls.  Errors as
 * for qmlp_forward_layers; QMLP_ERR_UNSUPPORTED for bfloat16.
 */
size_t qmlp_batch_workspace_bytes(const qmlp_mlp *layers, int L, int M, qmlp_dtype dtype);

qmlp_status qmlp_forward_batch(const qmlp_mlp *layers, int L, const void *x, int M,
                               qmlp_dtype dtype, void *y, void *ws, size_t ws_bytes,
                               qmlp_stream stream);

/*
 * L independent group-quantized linears of one shape, y_l = W_l x_l (Sec. 3.3:
 * every linear outside gate/up is INT4 in W4/W2-GateUp; at 2 bits they are
 * the uniform-W2 comparison point of Sec. 5.2): the attention projections of
 * a decoder layer (q, k and v as one [q+2kv][d] matrix, o) and the LM head.
 * w[0..L-1] are host descriptors of one shape [n][k] and width (4, or 2 with
 * group 64/128), 1 <= L <= 40; x [L][M][k] and y [L][M][n] binary16,
 * 1 <= M <= 16 (M == 0 is a no-op).  One launch over the batch, no workspace:
 * from two tokens on (2-bit rows of k <= 512: mostly from three) on the matrix
 * cores where a row fits one workgroup (k <= 6144, k <= 12288 at up to eight tokens, half of each at 4 bits in groups of
 * 32), else the stand-alone down kernel, which at several tokens takes
 * several times as long.  n % 64 == 0, k % 64 == 0.
 */
qmlp_status qmlp_linear_batch(const qmlp_qweight *w, int L, const void *x, int M,
                              qmlp_dtype dtype, void *y, qmlp_stream stream);

/*
 * A quantized linear with low-rank adapters of many requests beside it
 * (Sec. 3.1 Eq. (1) with an adapter per row; Sec. 4.2: the adapters stay
 * separate from the quantized base, so requests share it):
 *     y[m] = W x[m] + s_a B_a (A_a x[m]),   a = ids[m].
 * A [count][rank][k] and B [count][n][rank] in the activation type (adapters
 * of a lower rank are padded with zeros), scale fp32 [count] (NULL: 1.0), ids
 * int32 [M], all on the device.  A row whose id lies outside [0, count) has no
 * adapter and gets W x.  rank 8, 16, 32 or 64.  `adapters` may be NULL or have
 * count 0: W x alone (ids may then be NULL).
 */
typedef struct {
    const void *A;          /* [count][rank][k] activation type, 16-byte aligned */
    const void *B;          /* [count][n][rank] */
    const float *scale;     /* [count], or NULL */
    int32_t count, rank;
} qmlp_adapters;

/*
 * w: 2 or 4 bits, any group, k % 64 == 0, any n.  x [M][k] and y [M][n] are
 * binary16 or bfloat16, 0 <= M <= 2^20, with rows ldx >= k (a multiple of 8)
 * and ldy >= n elements apart; elements between the rows are neither read into
 * a result nor written.  t = A x is formed in one launch (with bfloat16 rows
 * rewritten as binary16 times a power of two per row, which keeps every element
 * down to 2^-28 of its row's largest exactly; a row that holds an infinity or
 * NaN, or whose adapter does, or whose t overflows fp32, gives infinities or
 * NaNs, and so may a bfloat16 row of more than 16 whose adapter's term exceeds
 * 2^113 times its largest element), the linear in a second: up to 16 rows with
 * weights as exact codes, more as a dense product of weights rounded once to
 * binary16, whose shares of k and adapters a third launch adds up where tiles
 * are few, or whose rows of many adapters one between the two prepares.
 * ws/ws_bytes: at least qmlp_linear_lora_workspace_bytes(...) of this or any
 * larger number of rows, any contents, nothing is kept between calls; one call
 * at a time per workspace.
 * M == 0 enqueues nothing.  Nothing is written outside y's M rows and ws.
 */
size_t qmlp_linear_lora_workspace_bytes(const qmlp_qweight *w, const qmlp_adapters *adapters, int M,
                                        qmlp_dtype dtype);

qmlp_status qmlp_linear_lora(const qmlp_qweight *w, const qmlp_adapters *adapters, const int32_t *ids,
                             const void *x, int64_t ldx, int M, qmlp_dtype dtype, void *y, int64_t ldy,
                             void *ws, size_t ws_bytes, qmlp_stream stream);

/*
 * The MLP of a mixture-of-experts decoder layer at decode (Sec. 5: the
 * routed experts of the GPT-OSS-20B-class model; only the routed experts'
 * weights are read per token): each of E experts is one block of
 * qmlp_forward (W4/W2-GateUp with its own adapters, or any width qmlp_mlp
 * lists), and token m's output is
 *     y[m] = sum_j topk_w[m][j] * expert_{topk_idx[m][j]}(x[m]).
 * experts[0..E-1]: host descriptors of one shape, 1 <= E <= 40.  x [M][d],
 * y [M][d] binary16; topk_idx int32 [M][k] and topk_w fp32 [M][k] are DEVICE
 * arrays (routing runs on the GPU); ids outside [0, E) are a precondition
 * violation (the kernels clamp them, so nothing is read outside the
 * table).  1 <= k <= E, M <= 16, M*k <= 40.  Every (token, slot) pair runs
 * as one instance.  Where tokens share enough experts that reading each
 * expert in use once saves more than its launches cost, the layer runs on the
 * matrix cores: LoRA-A, gate/up and down over the experts in use, their
 * instances side by side, and a combine launch over the instances' fp32
 * outputs.  Otherwise an expert chosen by two tokens is read twice, in two
 * launches over the M*k instances: gate/up, whose first workgroups of each
 * instance compute LoRA-A (with adapters) and hand t to the others as tagged
 * words, then down.  With
 * k <= 4 (and h of the k instances within the down kernel's LDS staging)
 * the down launch also forms y: one workgroup computes all k instances of
 * its output rows and adds them in fp32, w[m][j] y_j from j = 0, rounding
 * once to binary16.  Otherwise each instance's output is rounded to
 * binary16 and a combine launch adds them in the same order.
 * ws/ws_bytes: at least qmlp_moe_workspace_bytes(...): a 1024-byte control
 * block (uint32 words on 128-byte lines: word 0 counts the calls and tags
 * each call's t words, word 160 holds sticky error bits, 1 = a wait for t
 * gave up), t as tagged 64-bit words [M*k][2r], h and the per-instance
 * outputs (fp32 on the matrix cores).  The workspace must be ZERO before its first call, and zeroed
 * again after a call failed or an error bit appeared (the results of that
 * call are invalid).  One workspace serves one call at a time: calls that
 * overlap in time on the same workspace race.
 */
size_t qmlp_moe_workspace_bytes(const qmlp_mlp *experts, int E, int M, int k, qmlp_dtype dtype);

qmlp_status qmlp_forward_moe(const qmlp_mlp *experts, int E, const void *x, int M,
                             qmlp_dtype dtype, const int32_t *topk_idx, const float *topk_w, int k,
                             void *y, void *ws, size_t ws_bytes, qmlp_stream stream);

/* Launch shape of qmlp_forward_moe's weight launches for M tokens with k
 * routed experts each (M k instances) of a [d][f] expert, on a device with
 * `cus` compute units: the lanes per row of the gate/up launch (gu_bits 2 or
 * 4) and of the down launch (dn_bits 2 or 4).  Gate/up: a few instances
 * leave the chip with fewer than two workgroups per compute unit at the
 * usual choice, so the lanes per row double (more, shorter rows per
 * workgroup) until it has them.  Returns 2 when down also forms the routing
 * sum (k <= 4; the fewest lanes with at most three 16-byte units each),
 * 1 when it takes the pipelined kernel and a combine launch follows, 0 the
 * plain kernel; -1 for arguments outside d, f > 0 and multiples of 64,
 * M, k >= 1, M k <= 40, cus >= 1, non-null outputs.  Host-only. */
int qmlp_moe_lanes(int d, int f, int gu_bits, int dn_bits, int M, int k, int cus,
                   int *gu_lanes, int *dn_lanes);

/*
 * The router of a mixture-of-experts layer (Sec. 5: the routed experts of the
 * MoE decoder): l = x Wr^T + bias for x [M][d] and Wr [E][d] of one activation
 * type and bias fp32 [E] (or NULL), the k largest of each token in descending
 * order -- ties to the lower expert -- and their weights:
 *   TOPK_SOFTMAX  softmax of the k chosen logits;
 *   SOFTMAX       softmax over all E logits, taken at the chosen (not
 *                 normalised again);
 *   SIGMOID       sigmoid(l) over the sum of the k chosen sigmoids.
 * The choice is that of logits summed in fp64 (products of two 16-bit floats are
 * exact there), so it does not depend on how the work was split.  For many
 * tokens only the logits that could change places are formed so; the others, and
 * with them the weights, carry the rounding of fp32 sums of 32 products each, at
 * most 2^-18 |x| |w| of a logit and ordinarily 2^-23 of it.  An expert whose logit
 * is NaN or -inf (a bias of -inf masks it) is never chosen; +inf counts as the
 * largest fp32.  Where fewer than k experts are left, the remaining slots hold
 * expert -1 and weight 0.  topk_idx int32 [M][k] and topk_w fp32 [M][k] are what
 * qmlp_forward_moe takes (it clamps a -1, whose weight is 0).
 * 1 <= k <= 16, k <= E <= 512, d % 8 == 0, 0 <= M <= 2^20 (0: nothing to do).
 * ws: qmlp_moe_route_workspace_bytes(E, M) bytes, any contents, nothing kept
 * between calls; one call at a time per workspace.
 */
typedef enum { QMLP_SCORE_TOPK_SOFTMAX = 0, QMLP_SCORE_SOFTMAX = 1, QMLP_SCORE_SIGMOID = 2 } qmlp_score;

size_t qmlp_moe_route_workspace_bytes(int E, int M);

qmlp_status qmlp_moe_route(const void *router, const float *bias, const void *x, int M, int d, int E, int k,
                           qmlp_score score, qmlp_dtype dtype, int32_t *topk_idx, float *topk_w, void *ws,
                           size_t ws_bytes, qmlp_stream stream);

/*
 * A whole mixture-of-experts layer for a few tokens (Sec. 5, Sec. 3.3, Sec.
 * 4.2): the router above, then y[m] = sum_j w[m][j] expert_{idx[m][j]}(x[m]) with
 * each expert a gated MLP of qmlp_forward with its own adapters.
 * `mlp` holds the experts one after another: gate and up [E f][d], down
 * [E d][f], A_gate/A_up [E][rank][d], B_gate/B_up [E][f][rank] (n_out E f, E f
 * and E d; a packed matrix of stacked rows is the stack of packed matrices).
 * Gate/up 2 or 4 bits and down 4 or 2 bits, groups of 32, 64 or 128, d and f
 * multiples of 64, rank 0, 8, 16 or 32, E <= 512, topk <= 16.  Binary16, 0 <= M
 * <= 64 (0: nothing to do).  A token none of whose experts can be chosen gets
 * zeros.  h is rounded to binary16; the experts' outputs stay fp32 until the
 * weighted sum, slots in order, is rounded once.
 * ws: qmlp_moe_layer_workspace_bytes(...) bytes, any contents, nothing kept
 * between calls; one call at a time per workspace.
 * Up to four tokens of at most 40 experts qmlp_moe_route and qmlp_forward_moe
 * are the faster way (one token of the 20B-class layer 26.9 us, here 35.2).
 */
typedef struct {
    const void *router;      /* [E][d] binary16, 16-byte aligned */
    const float *bias;       /* [E] or NULL */
    int32_t experts, topk, score;
    qmlp_mlp mlp;
} qmlp_moe;

size_t qmlp_moe_layer_workspace_bytes(const qmlp_moe *layer, int M, qmlp_dtype dtype);

qmlp_status qmlp_moe_layer(const qmlp_moe *layer, const void *x, int M, qmlp_dtype dtype, void *y, void *ws,
                           size_t ws_bytes, qmlp_stream stream);

/* ------------------------- attention over a cache of keys and values in 4 bits */

/*
 * What lies between a decoder layer's q/k/v projection (qmlp_linear_batch,
 * qmlp_linear_lora) and its output projection, for a batch of requests whose
 * keys and values stay in a paged cache: the pages of a step's tokens
 * (qmlp_kv_plan), norm, rotation and the write (qmlp_qk_norm_rope), attention
 * (qmlp_kv_attention).  Every array is on the device and nothing is read on
 * the host, so a decoding step, its growth by new pages included, can be
 * captured once and replayed.
 *
 * Storage format of the cache.  A page holds `page` tokens of one layer:
 *   data [pages][kv_heads][2][page * (head_dim/2 + 4)] bytes, K then V: the
 * codes of the page's tokens, then binary16 (scale, zero) of each.  One group is
 * one token's head_dim numbers of one head; its quantizer is that of the
 * weights at b = 4 (scale and zero as above, value scale * (code - zero)); a
 * group that holds an infinity or NaN, or whose scale passes 65504, is stored as
 * scale NaN, zero 0, codes 0 and reads back as NaN.  Eight codes are a 32-bit
 * word: dims 8w + 0..7 at nibbles 0, 4, 1, 5, 2, 6, 3, 7 of word w.  Words of K
 * are [token][head_dim/8]; words of V [token / 4][head_dim/8][token % 4].
 * A slot is page number * page + place in the page; -1 is no slot.
 * head_dim 64 or 128; page 16, 32, 64, 128 or 256; fewer than 2^31 slots.
 */
typedef struct {
    void *data;             /* qmlp_kv_cache_bytes() bytes, 16-byte aligned */
    int32_t pages, kv_heads, head_dim, page;
} qmlp_kv_cache;

/* Bytes of a cache; 0 for one that is not supported. */
size_t qmlp_kv_cache_bytes(int pages, int kv_heads, int head_dim, int page);

/*
 * The pages of one step.  Request b has lens[b] tokens in the cache and adds
 * new_tokens[b]; -1 (or less) ends it.  table [B][W] holds each request's page
 * numbers in order; free_pages [N] is a stack of unused pages with n_free[0] of
 * them.  In this order:
 *  1. the pages of ended requests, ceil(lens/page) each, are pushed on the
 *     stack, requests and their pages in order (what would pass N is dropped);
 *  2. a growing request that lacks pages takes them from the top of the stack,
 *     requests in order, page after page, into its row of the table.  A request gets all it needs or is
 *     refused: it is refused if its tokens would pass W pages, if the step's tokens up to
 *     its last pass `tokens`, or if what it and those before it need (the
 *     ones that lacked pages counted) passes the stack.
 * starts [B+1]: the first token of each request among the step's, the sums of
 * the new tokens (refused ones too, ended ones none; at most 2^31 - 1).  positions and
 * slots [tokens]: place in its request and slot of every token; slot -1 for
 * the tokens of refused requests and of pages whose slots are not in [0, 2^31); past the last token position 0, slot -1.
 * lens_out [B]: lens + new, lens for a refused request, 0 for an ended one.
 * n_free_out[0]; short_out[0]: requests refused.  lens_out may be lens and
 * n_free_out may be n_free (a chain of steps); otherwise no two arrays overlap.
 * Entries of the table past a request's pages are left as they are, those of an
 * ended request too, and stack places that nothing is pushed to: the same
 * call on the same lens and n_free gives the same again.
 * lens outside [0, W page] and n_free outside [0, N] are taken as the nearest number inside.
 * 0 <= B <= 2048, 1 <= W <= 2^20, W * page <= 2^30, 0 <= N, 0 <= tokens <= 2^24.  One launch
 * (none with B = 0: nothing is written).
 */
typedef struct {
    const int32_t *lens, *new_tokens;   /* [B] */
    int32_t *table, *free_pages;        /* [B][W], [N] */
    const int32_t *n_free;              /* [1] */
    int32_t *slots, *positions;         /* [tokens] */
    int32_t *starts;                    /* [B+1] */
    int32_t *lens_out, *n_free_out, *short_out;     /* [B], [1], [1] */
    int32_t B, page, W, N, tokens;
} qmlp_plan;

qmlp_status qmlp_kv_plan(const qmlp_plan *p, qmlp_stream stream);

/* Which dims of a head turn together: (i, i + rot/2), or (2i, 2i + 1). */
typedef enum { QMLP_PAIRS_HALF = 0, QMLP_PAIRS_NEXT = 1 } qmlp_pairs;

/*
 * Queries and keys of T tokens, one launch: each head x of q and k becomes
 *   u = x / sqrt(mean(x^2) + eps) * weight      (weight NULL: u = x),
 *   (u_i, u_j) -> mul (u_i cos a - u_j sin a, u_j cos a + u_i sin a) with
 *   a = positions[t] inv_freq[p] for the p-th pair of the first `rot` dims
 *   (inv_freq NULL: no rotation),
 * rounded to the activation type (q once, k to fp32 first); q goes to q_out, k to k_out (or NULL)
 * and, with a cache, k and v of the tokens with a slot in [0, slots of the cache)
 * are quantized from the activation type and written there.  q, k and v are
 * rows ldq, ldk, ldv elements apart with their heads side by side (views of one
 * q/k/v row, for instance).  q_out may be q and k_out may be k, at the same
 * address and stride; otherwise outputs overlap nothing.  q arithmetic is fp32 (fp64 for heads whose
 * mean square leaves 2^-100 .. 2^120) and k's fp64 (a code hangs on the last bits of numbers next to a border), angles are
 * reduced in fp64.
 */
typedef struct {
    const void *q, *k, *v;              /* [T][heads or kv_heads][head_dim], 16-byte aligned; v only with a cache */
    int64_t ldq, ldk, ldv;              /* elements from row to row, multiples of 8 */
    void *q_out, *k_out;
    int64_t ldq_out, ldk_out;
    const void *q_weight, *k_weight;    /* [head_dim] activation type, 16-byte aligned, or NULL */
    const int32_t *positions;           /* [T] (with inv_freq) */
    const float *inv_freq;              /* [rot/2], or NULL */
    const int32_t *slots;               /* [T] (with a cache) */
    int32_t heads, kv_heads, head_dim;  /* head_dim 64 or 128; heads may be 0 (q and q_out unused) */
    int32_t rot;                        /* a multiple of 16, 16 .. head_dim (with inv_freq) */
    int32_t pairs;                      /* qmlp_pairs */
    float eps, mul;                     /* eps >= 0 */
} qmlp_heads;

/* cache may be NULL (k_out then receives k).  0 <= T <= 2^20.  Two tokens with the same
 * slot leave a mixture of the two there. */
qmlp_status qmlp_qk_norm_rope(const qmlp_heads *h, int T, qmlp_dtype dtype, const qmlp_kv_cache *cache,
                              qmlp_stream stream);

/* What the cache holds at slots [T]: k and v [T][kv_heads][head_dim] (either may be
 * NULL) rounded once to the type (past its largest number: infinity); zeros for a slot outside the
 * cache.  T * kv_heads at most 2^27. */
qmlp_status qmlp_kv_read(const qmlp_kv_cache *cache, const int32_t *slots, int T, qmlp_dtype dtype, void *k, void *v,
                         qmlp_stream stream);

/*
 * Causal attention of a step's tokens over the cached keys and values, their
 * own among them.  Request b has lens[b] tokens in the cache, the last n =
 * starts[b+1] - starts[b] of them this step's: rows starts[b] + i of q and y,
 * at position p = lens[b] - n + i (starts NULL: T == B and one row each).
 * Head g reads K/V head g / (heads / kv_heads):
 *   y = sum_j w_j V_j / (sum_j w_j + exp(sinks[g])),  w_j = exp(scale q . K_j),
 * j over max(0, p - window + 1) .. p (window 0: from 0), sinks NULL: no such term.
 * A row that sees nothing is zeros.  A page number outside the cache hides its tokens.
 * table [B][W]; lens past W pages count as W pages.  q and y [T][heads][head_dim] in
 * rows ldq and ldy elements apart, y overlapping nothing.  Rows of y before starts[0] and from starts[B] on
 * are left as they are (starts has to be rising, 0 <= starts <= T; rows past T are not touched).
 * Codes enter the products as exact integers; scores, sums and outputs are fp32; weights times the
 * value's scale are rounded to binary16, with a power of two that keeps 2^-22 of the largest normal (where a row's largest score
 * passes 2^20 in size, it weighs 1).  Scores past fp32 make their rows NaN (zeros, where all of a row's are -infinity).
 * bfloat16 queries enter them as binary16 times a power of two: a number of a row loses at most 2^-27 of the row's
 * largest, whatever the other rows hold.
 * Keys or values that are NaN, and rows of q with an infinity or NaN, make the rows that
 * see them NaN and no others.
 * max_new: the most new tokens of any request, as far as the host knows.  It chooses kernels and sizes
 * the workspace; a request with more is computed all the same, slower.
 * heads a multiple of kv_heads, 0 <= B <= 2048, 0 <= T <= 2^20, 1 <= W, W * page <= 2^30, scale finite,
 * window >= 0.
 * ws: qmlp_kv_attention_workspace_bytes(...) of this or a larger max_new, ZERO before its first call (and after
 * a call that failed); each call leaves it ready for the next, of any shape it is large enough for.  One call at
 * a time per workspace.
 */
typedef struct {
    const void *q;                      /* [T][heads][head_dim], 16-byte aligned */
    void *y;                            /* the same */
    int64_t ldq, ldy;                   /* elements from row to row, multiples of 8 */
    const int32_t *table, *lens, *starts;       /* [B][W], [B], [B+1] or NULL */
    const float *sinks;                 /* [heads] or NULL */
    void *ws;
    size_t ws_bytes;
    int32_t T, heads, B, W, max_new, window;
    float scale;
} qmlp_attention;

size_t qmlp_kv_attention_workspace_bytes(const qmlp_kv_cache *cache, int heads, int max_new);

qmlp_status qmlp_kv_attention(const qmlp_kv_cache *cache, const qmlp_attention *a, qmlp_dtype dtype, qmlp_stream stream);

/* ---------------------------------------------- inspection (not timed) */

/*
 * Unpack a packed matrix into canonical form: codes uint8 [n][k] and the
 * binary16 bits of scale and zero [n][k/g] (QDQ view, Sec. 6.3).
 */
qmlp_status qmlp_unpack(const qmlp_qweight *w, uint8_t *codes, uint16_t *scales,
                        uint16_t *zeros, qmlp_stream stream);

/* The dequantized weight scale * (q - zero), rounded once to binary16
 * (nearest-even; q == zero gives +0), [n][k] row-major. */
qmlp_status qmlp_dequant(const qmlp_qweight *w, uint16_t *w_f16, qmlp_stream stream);

/* Number of kernel launches qmlp_forward makes for this block at M tokens:
 * 1 when the whole layer runs as one fused kernel (the decode shapes it
 * covers), 2 or 3 when it runs as the LoRA-A, gate/up and down kernels in
 * stream order; a bfloat16 prefill chunk makes LoRA-A and its reduction
 * (with an adapter), gate/up, down, and, when down splits f into slices (f a
 * multiple of 128, and the slices' workgroups stay within about one round
 * over the compute units), the slices' reduction; 0 if the call would be rejected.  Host-only,
 * enqueues nothing. */
int qmlp_forward_launches(const qmlp_mlp *mlp, int M, qmlp_dtype dtype);

/* Measurement hook (not part of the MLP): read `bytes` of device memory at
 * `buf` once with 128-bit loads -- the non-temporal form the weight stream
 * uses when `nontemporal` is nonzero, plain loads otherwise -- and write one
 * XOR word per wave to out[0 .. 4*blocks).  Decode is bound by the rate of
 * loading weights (Sec. 1, Sec. 3.3); this kernel does nothing but load, so
 * its duration is the HBM read rate this GPU sustains, and its byte
 * counters against the known size calibrate the counters of the decode
 * kernels.  One launch of `blocks` 256-thread workgroups.  bytes % 16 == 0,
 * 1 <= blocks <= 65536, buf 16-byte aligned, out 4-byte aligned. */
qmlp_status qmlp_probe_stream_read(const void *buf, size_t bytes, uint32_t *out, int blocks,
                                   int nontemporal, qmlp_stream stream);

/* A static, human-readable name of a status code. */
const char *qmlp_status_string(qmlp_status s);

#ifdef __cplusplus
}
#endif

#endif /* QMLP_H */
