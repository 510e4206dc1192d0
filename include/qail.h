/*
 * qail.h - C ABI of libqail: 4-bit quantised linear layers on AMD MI355X (gfx950).
 *
 * The operations are the deployed low-bit layers behind the efficiency results
 * of "Quantization-Aware Imitation-Learning for Resource-Efficient Robotic
 * Control" (Sec. 5.4 "Implementation" and the appendix "Analysis"):
 *
 *   W4A16  weight-only 4-bit linears of the Llama-2-7B backbone of the VLA
 *          policy.  Sec. 2.1: LLM linears are limited by weight loading, so only
 *          the weight operand of the GEMM is quantised; Sec. 5.1: 4-bit AWQ
 *          format (unsigned codes, scale, integer zero-point).  The appendix
 *          "Analysis" finds the decode stage memory-bound; that is the M = 1 case.
 *   W4A4   4-bit weights and 4-bit activations of the ResNet encoder of the
 *          driving policy.  Sec. 2.1: convolutional models are compute-bound, so
 *          both GEMM operands are quantised; Sec. 5.1: RTN / LSQ integer format.
 *
 * Conventions for every call
 *   - All data pointers are DEVICE pointers into memory owned by the caller,
 *     16-byte aligned.  Descriptors and size outputs are HOST pointers.  The
 *     library allocates nothing and frees nothing.  The only state it keeps is
 *     what it learns about the device at a call's first use (the number of
 *     compute units, the opt-in for large LDS blocks); those are set once,
 *     through atomics, so calls may come from several host threads.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     A call validates its arguments, enqueues its kernels and returns; it never
 *     synchronises.  Outputs are fully overwritten.
 *   - Argument errors (null pointer, bad shape, misalignment, short workspace)
 *     are detected before anything is launched and leave device memory untouched;
 *     they can be exercised on a host without a GPU.  A failed launch maps to
 *     QAIL_ERR_HIP.
 *   - Packed 4-bit data: 8 codes per uint32, code j of the packed axis in bits
 *     [4*(j%8), 4*(j%8)+3] of word j/8.  Signed codes are two's-complement nibbles.
 *   - bf16 and fp16 values cross the boundary as their 16-bit patterns (uint16_t).
 *   - Inputs are finite.  NaN or infinity in a tensor to be quantised gives
 *     unspecified codes (no fault).
 */
#ifndef QAIL_H
#define QAIL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    QAIL_OK = 0,
    QAIL_ERR_NULL = -1,        /* a required pointer is NULL */
    QAIL_ERR_SHAPE = -2,       /* a dimension is non-positive or violates a divisibility rule */
    QAIL_ERR_ALIGN = -3,       /* a device pointer is not 16-byte aligned */
    QAIL_ERR_WORKSPACE = -4,   /* workspace missing or smaller than the matching *_workspace query */
    QAIL_ERR_UNSUPPORTED = -5, /* valid request outside what the kernels cover */
    QAIL_ERR_HIP = -6          /* the HIP runtime refused a launch */
} qail_status;

typedef enum {
    /* Unsigned codes 0..15, one fp16 scale and one integer zero-point 0..15 per
     * group of `group_size` consecutive k of a row (Sec. 5.1, VLA policy;
     * group_size == K is the channel-wise case of the appendix). */
    QAIL_W4_ASYM_GROUP = 0,
    /* Signed codes -8..7, one fp32 scale per row (output channel); group_size is
     * ignored (Sec. 5.1, driving policy). */
    QAIL_W4_SYM_CHANNEL = 1,
    /* 8-bit variants (Sec. 5.4: W8A8 driving encoder, 8-bit weight-only backbone).  The paper
     * names no 8-bit quantiser; both are symmetric round-to-nearest with signed codes
     * -127..127, packed 4 per word (code i of a word in bits 8*(i%4)..8*(i%4)+7):
     * one fp32 scale max|w|/127 per row ... */
    QAIL_W8_SYM_CHANNEL = 2,
    /* ... or one fp16 scale per group of `group_size` consecutive k, rounded up, >= 2^-14. */
    QAIL_W8_SYM_GROUP = 3
} qail_scheme;

/* A quantised weight matrix W[N][K] (row n = output channel, K contiguous). */
typedef struct {
    int32_t N;          /* rows / output channels, >= 1 */
    int32_t K;          /* columns / input channels, multiple of 8 */
    int32_t group_size; /* ASYM_GROUP: multiple of 8 that divides K */
    int32_t scheme;     /* qail_scheme */
} qail_wdesc;

/* A 2-D convolution read as a GEMM with M = B*OH*OW, N = Cout, K = KH*KW*Cin,
 * OH = (H + 2*pad - KH)/stride + 1 (same for OW).  KH = KW = 1, stride = 1,
 * pad = 0 makes it a plain [B*H*W, Cin] x [Cout, Cin]^T GEMM. */
typedef struct {
    int32_t B, H, W;    /* batch, input height, input width */
    int32_t Cin, Cout;  /* Cin multiple of 8; Cout >= 1 */
    int32_t KH, KW;     /* filter taps */
    int32_t stride, pad;
} qail_conv_desc;

int qail_version(void);
const char* qail_status_string(int status);

/* ---------------------------------------------------------------- quantise --
 * Sec. 2.1 (round-to-nearest) and Sec. 5.1 (the two 4-bit formats). */

/* Byte sizes of the packed form of `d` (host computation only):
 *   qweight  N * K/8 uint32
 *   scales   ASYM_GROUP: N * K/group_size fp16     SYM_CHANNEL: N fp32
 *   zeros    ASYM_GROUP: N * ceil(K/group_size/8) uint32 (unused nibbles 0)
 *            SYM_CHANNEL: 0
 * Any output pointer may be NULL. */
int qail_packed_sizes(const qail_wdesc* d, size_t* qweight_bytes, size_t* scales_bytes,
                      size_t* zeros_bytes);

/* Round-to-nearest quantisation of w (fp32, [N][K] row-major) into the packed form.
 *
 * ASYM_GROUP, per row and group, in IEEE fp32 with correctly rounded division:
 *   lo = min(min w, 0); hi = max(max w, 0)
 *   s  = (hi - lo)/15 rounded UP to fp16, at least 2^-14; an all-zero group has s = 1
 *   z  = clamp(rint(-lo/s), 0, 15);  q = clamp(rint(w/s) + z, 0, 15)   (ties to even)
 * SYM_CHANNEL, per row:
 *   s  = max|w|/7 (fp32; 1 for an all-zero row);  q = clamp(rint(w/s), -8, 7)
 *   `zeros` is ignored and may be NULL.
 *
 * range_errors (device, one uint32, may be NULL): if given it is NOT cleared; it is
 * incremented once per ASYM group whose (hi-lo)/15 exceeds the largest fp16
 * (65504).  Such a group is stored with s = 65504 and clamped codes. */
int qail_quantize_weights(const qail_wdesc* d, const float* w, uint32_t* qweight, void* scales,
                          uint32_t* zeros, uint32_t* range_errors, void* stream);

/* Packed words -> one code per byte, [N][K]: uint8 0..15 (ASYM_GROUP) or int8 -8..7
 * (SYM_CHANNEL, sign-extended). */
int qail_unpack_weights(const qail_wdesc* d, const uint32_t* qweight, uint8_t* codes, void* stream);

/* One activation step size for a whole tensor (appendix: tensor-wise activation
 * quantisation): *s_a = max(a)/15 in fp32, or 1 if no element is positive.
 * a: fp32 [n]; s_a: device, one float. */
int qail_act_scale_u4(const float* a, size_t n, float* s_a, void* stream);

/* q = clamp(rint(a / *s_a), 0, 15), packed 8 per word along the flat index
 * (for an NHWC tensor that is along C).  n multiple of 8; s_a: device, one float. */
int qail_quantize_act_u4(const float* a, size_t n, const float* s_a, uint32_t* a_u4, void* stream);

/* ------------------------------------------------------------------ W4A16 --
 * y[m][n] = sum_k x[m][k] * (q[n][k] - z[n][k/g]) * s[n][k/g]
 * Sec. 2.1 (weight-only quantised GEMM operand); appendix "Analysis" (decode is
 * the memory-bound stage, prefill the compute-heavy one). */

/* Bytes of device scratch the call below needs for this (d, M).  0 for the streaming
 * kernels (M <= 16 on shapes they take, M <= 32 at group_size 128 with an even number of
 * groups per row); for shapes of the matrix-core GEMM it holds (also at M <= 64, where another
 * kernel may be faster for them and uses none) an fp16 copy
 * of x (rows padded to a multiple of 128, K to a multiple of 128), one float per padded
 * row and per output column, and two tile-shaped fp32 slots per block of the grid (one
 * block per compute unit) for output tiles whose K range is shared between blocks (tens
 * of MB at prefill sizes).  The workspace must be 256-byte aligned, is
 * overwritten by every call and carries nothing between calls; calls that share one
 * must be ordered on one stream. */
int qail_w4a16_workspace(const qail_wdesc* d, int32_t M, size_t* bytes);

/* d must be ASYM_GROUP.  x: bf16 [M][K]; y: bf16 [M][N].  Products are accumulated
 * in fp32 and rounded once to bf16 (nearest even).  M = 1 (decode) is served by a
 * bandwidth-bound streaming kernel, 2 <= M <= 4 by the same stream with four rows of x,
 * up to M = 16 (M = 32 at group_size 128 with an even number of groups per row) by a
 * weight-streaming MFMA kernel (x and codes exact in the products; an x beyond 2e36 may
 * overflow a sum of codes times x on the way),
 * 5 <= M <= 64 at group_size 128 or 64 with K % 128 == 0 and an even number of groups per row, where
 * that was measured to be faster, by a kernel with one pass over K (the same products, any finite x),
 * larger M (prefill) and other shapes by an fp16 MFMA kernel that expands the codes in registers
 * ((q - z) * s rounded once to fp16, x rescaled per row by a power of two).
 * workspace may be NULL when the query returns 0; otherwise a missing or short one
 * is QAIL_ERR_WORKSPACE and a misaligned one QAIL_ERR_ALIGN. */
int qail_w4a16_linear(const qail_wdesc* d, const uint32_t* qweight, const uint16_t* scales,
                      const uint32_t* zeros, const uint16_t* x, uint16_t* y, int32_t M,
                      void* workspace, size_t workspace_bytes, void* stream);

/* One linear of a batch for qail_w4a16_linear_batch. */
typedef struct {
    qail_wdesc d;
    const uint32_t* qweight;
    const uint16_t* scales;
    const uint32_t* zeros;
    const uint16_t* x;   /* bf16 [M][K] */
    uint16_t* y;         /* bf16 [M][N] */
} qail_w4a16_item;

/* `count` linears with the same M, given as a HOST array, enqueued on one stream
 * (appendix "Analysis": a decode step is a fixed sequence of such linears, 4 per
 * layer).  The items must be independent: no item may read what another writes.
 * The library may run them in fewer launches, items side by side on shares of the
 * GPU.  The result is that of `count` calls of qail_w4a16_linear: bit for bit for
 * M <= 4; for larger M an item's sum over K may be divided between waves or blocks
 * at other places than in a call of its own, so the two can differ by the rounding
 * of fp32 partial sums (far inside the W4A16 tolerance); the same call on the same
 * GPU always gives the same bits.  count >= 0 (0 is a no-op). */
int qail_w4a16_linear_batch(const qail_w4a16_item* items, int32_t count, int32_t M,
                            void* workspace, size_t workspace_bytes, void* stream);
/* Workspace for the batch call.  Items that share a launch (M > 16: up to 8 at a time)
 * keep their prepared activations side by side in it, so the need can exceed that of
 * any single item; launches that follow each other on the stream reuse it. */
int qail_w4a16_batch_workspace(const qail_w4a16_item* items, int32_t count, int32_t M,
                               size_t* bytes);

/* Linears that depend on each other, M = 1, in one launch (appendix "Analysis": the decode stage
 * walks the backbone's linears one after the other, each a bandwidth-bound stream of weights).
 * Item i + 1 does not read its x before every element of item i's y has been written, so x of
 * item i + 1 may be, or overlap, y of item i; apart from that the results are those of
 * qail_w4a16_linear_batch at M = 1, bit for bit.  The whole grid is resident on the GPU and the
 * blocks meet between two items through counters in the workspace, while the first weights of the
 * next item are already on their way: the stream of weights does not stop between items as it
 * does between launches.  Up to 32 items share a launch; longer lists take several.
 *   items      HOST array; every item must be one the M = 1 streaming kernel takes
 *              (K % 32 == 0, group_size % 32 == 0, K <= 12288) with N <= 512 * CUs, else
 *              QAIL_ERR_UNSUPPORTED.
 *   workspace  qail_w4a16_chain_workspace() bytes, 256-byte aligned.  Its first uint32 is a status
 *              word, written by the call: 0 if every block saw the others arrive, 1 if some block
 *              gave up waiting (possible only when other work keeps part of the grid off the GPU;
 *              the outputs are then unspecified, and every kernel still ends). */
int qail_w4a16_chain_workspace(const qail_w4a16_item* items, int32_t count, size_t* bytes);
int qail_w4a16_linear_chain(const qail_w4a16_item* items, int32_t count, void* workspace,
                            size_t workspace_bytes, void* stream);

/* Low-rank adapter beside a 4-bit linear (Sec. 5.1: the 4-bit policy is fine-tuned with
 * rank-32 adapters on the quantised backbone; they stay separate from the packed weights):
 *     y[m][n] = sum_k x[m][k] w_hat[n][k]  +  scaling * sum_j (sum_k x[m][k] A[j][k]) B[n][j]
 * A: bf16 [r][K], B: bf16 [N][r], device memory, 16-byte aligned; 8 <= r <= 64, r % 8 == 0. */
typedef struct {
    const uint16_t* A;
    const uint16_t* B;
    int32_t r;
    float scaling;
} qail_lora;

/* Like qail_w4a16_linear_batch with one adapter per item (loras: HOST array of `count`).
 * At M = 1 on shapes the streaming kernel takes, the up-projection joins the linear before
 * the single bf16 rounding of y; otherwise it is added to the rounded y and rounded again
 * (inside the W4A16 tolerance).  The workspace (query below; 256-byte aligned) holds the
 * linear's own workspace and the down-projections x A^T in fp32.  Errors as for the batch
 * call, plus QAIL_ERR_SHAPE for a rank outside the range above. */
int qail_w4a16_lora_workspace(const qail_w4a16_item* items, const qail_lora* loras, int32_t count,
                              int32_t M, size_t* bytes);
int qail_w4a16_linear_lora_batch(const qail_w4a16_item* items, const qail_lora* loras, int32_t count,
                                 int32_t M, void* workspace, size_t workspace_bytes, void* stream);

/* qail_w4a16_linear_lora_batch for callers that cannot allocate device memory (code under
 * HIP graph capture, serving loops that must not call hipMalloc, harnesses that forbid it):
 * the same kernels and the same results, with the workspace taken from a scratch array that is
 * part of the library's device image (qail_static_scratch_bytes: 1 MiB, held on every GPU the
 * library runs on until the process ends).  The call allocates nothing and frees nothing.
 * A request whose qail_w4a16_lora_workspace figure exceeds the scratch returns
 * QAIL_ERR_WORKSPACE before anything is launched (a decode batch of M <= 16 on up to 16
 * linears that the streaming kernels take, e.g. the 7B shapes with groups of 128, needs
 * 64 KiB; anything routed to the matrix-core GEMM needs megabytes and does not fit).  All calls on one GPU share that GPU's array: calls that
 * overlap on one GPU (two streams, two host threads) race on it and must be serialised by the
 * caller; calls that follow each other on one stream are safe, since each call writes what it
 * reads.  The scratch address of a GPU is looked up at the first call made with that GPU
 * current; make that first call outside graph capture. */
int qail_static_scratch_bytes(size_t* bytes);
int qail_w4a16_linear_lora_batch_static(const qail_w4a16_item* items, const qail_lora* loras,
                                        int32_t count, int32_t M, void* stream);

/* ------------------------------------------------------------------- W4A4 --
 * acc[(b,oh,ow)][n] = sum_{kh,kw,c} a[b][oh*stride+kh-pad][ow*stride+kw-pad][c] * w[n][kh][kw][c]
 * with zero outside the image, exact in int32; then optionally
 * y = float(acc) * scale[n] + bias[n]   (one fp32 fused multiply-add).
 * Sec. 2.1 (both GEMM operands quantised for compute-bound convolutions);
 * Sec. 5.4 (W4A4 GPU kernels of the driving policy). */

int qail_w4a4_workspace(const qail_conv_desc* d, size_t* bytes);

/* a_u4: packed unsigned codes, NHWC [B][H][W][Cin/8] words.
 * w_s4: packed signed codes [Cout][KH][KW][Cin/8] words.
 * acc_out: int32 [M][Cout] or NULL.  y_out: fp32 [M][Cout] or NULL (then scale and
 * bias, fp32 [Cout], are required).  At least one output must be given.
 * |acc| <= 8*15*K must stay below 2^27 (K <= 1118480). */
int qail_w4a4_gemm(const qail_conv_desc* d, const uint32_t* a_u4, const uint32_t* w_s4,
                   int32_t* acc_out, const float* scale, const float* bias, float* y_out,
                   void* workspace, size_t workspace_bytes, void* stream);

/* The same convolution with the output written directly as the NEXT layer's packed
 * unsigned 4-bit activations (Sec. 5.1 and the appendix's implementation details for
 * autonomous driving: every activation tensor of the driving encoder is 4-bit with one
 * step per tensor, so the consumer's step s_out is a constant of the network).  Per
 * output element, each line one correctly rounded fp32 operation (no fused multiply-add):
 *     t = float(acc) * scale[n]
 *     t = t + bias[n]
 *     t = t + r                  only with a shortcut, see below
 *     t = max(t, 0)              ReLU
 *     q = clamp(rint(t / s_out), 0, 15)        rint: ties to even
 * out_u4: [M][Cout/8] words, i.e. NHWC [B][OH][OW][Cout/8], the a_u4 layout; Cout % 8 == 0.
 * Shortcut of a residual block, at most one of
 *     res_u4:  packed unsigned codes [M][Cout/8] (the block input), r = res_scale * code;
 *     res_f32: fp32 [M][Cout] (a projection shortcut's y_out), r = res_f32[m][n].
 * scale, bias: fp32 [Cout], required.  s_out > 0 and res_scale >= 0 are host values.
 * All buffers are device memory owned by the caller; nothing is allocated, the call is
 * enqueued on `stream` and returns.  Errors as for qail_w4a4_gemm, plus QAIL_ERR_SHAPE for
 * Cout % 8 != 0, s_out not positive and finite, or two shortcuts at once. */
int qail_w4a4_conv_u4(const qail_conv_desc* d, const uint32_t* a_u4, const uint32_t* w_s4,
                      const float* scale, const float* bias, float s_out,
                      const uint32_t* res_u4, float res_scale, const float* res_f32,
                      uint32_t* out_u4, void* workspace, size_t workspace_bytes, void* stream);

/* Several independent W4A4 convolutions in as few launches as possible (one, when every
 * item is a shape the tiled kernel runs and count <= 4).  Sec. 5.1 / appendix: the driving
 * encoder is a ResNet, whose down-sampling blocks start with two convolutions that read the same
 * input, the 3x3 stride-2 one and the 1x1 projection of the shortcut; at a small batch a launch
 * costs more than either of them.
 * An item is the argument list of qail_w4a4_gemm (out_u4 == NULL: acc_out and / or y_out) or
 * of qail_w4a4_conv_u4 (out_u4 != NULL: acc_out and y_out must be NULL); every rule of those
 * two calls holds per item, and each item's results equal the single call's bit for bit.
 * Items must be independent: no item may read a buffer another item writes, and no two may
 * write the same one.  1 <= count <= 64.  Errors are reported before anything is launched. */
typedef struct {
    qail_conv_desc d;
    const uint32_t* a_u4;    /* device */
    const uint32_t* w_s4;    /* device */
    const float* scale;      /* device, fp32 [Cout]; required with y_out or out_u4 */
    const float* bias;       /* device, fp32 [Cout]; required with y_out or out_u4 */
    int32_t* acc_out;        /* device, int32 [M][Cout] or NULL */
    float* y_out;            /* device, fp32 [M][Cout] or NULL */
    uint32_t* out_u4;        /* device, [M][Cout/8] words or NULL */
    float s_out;             /* fused output only */
    float res_scale;         /* fused output with res_u4 only */
    const uint32_t* res_u4;  /* device or NULL */
    const float* res_f32;    /* device or NULL */
} qail_conv_item;
int qail_w4a4_conv_batch(const qail_conv_item* items, int32_t count, void* stream);

/* ------------------------------------------------------------------ 8-bit --
 * Sec. 5.4 deploys the driving encoder also as W8A8 and the backbone also with 8-bit
 * weights only.  Weights: qail_quantize_weights / qail_packed_sizes with the W8 schemes
 * (zeros unused, may be NULL; qail_unpack_weights is not needed: the codes are bytes). */

/* One activation step for a whole tensor: *s_a = max|a| / 127 in fp32, 1 if all zero. */
int qail_act_scale_s8(const float* a, size_t n, float* s_a, void* stream);

/* q = clamp(rint(a / *s_a), -127, 127), 4 codes per word along the flat index; n % 4 == 0. */
int qail_quantize_act_s8(const float* a, size_t n, const float* s_a, uint32_t* a_s8, void* stream);

/* qail_w4a4_gemm with signed 8-bit codes on both sides: a_s8 NHWC [B][H][W][Cin/4] words,
 * w_s8 [Cout][KH][KW][Cin/4] words, Cin % 4 == 0, K = KH*KW*Cin <= 131071 (int32 exact for
 * all codes in [-128, 127]).  Outputs, errors and ownership as for qail_w4a4_gemm. */
int qail_w8a8_gemm(const qail_conv_desc* d, const uint32_t* a_s8, const uint32_t* w_s8,
                   int32_t* acc_out, const float* scale, const float* bias, float* y_out,
                   void* workspace, size_t workspace_bytes, void* stream);

/* y[m][n] = sum_k x[m][k] * q[n][k] * s[n][k/g], d of scheme QAIL_W8_SYM_GROUP, x and y bf16,
 * fp32 accumulation, one rounding.  M = 1 runs a bandwidth-bound streaming kernel (K % 16 == 0,
 * group_size % 16 == 0, K + K/g <= 16384).  2 <= M <= 32 at group_size 128 with an even number
 * of groups per row (N * K below 2 GB) runs the small-batch streaming kernel of
 * qail_w4a16_linear with byte weights, or, as 33 <= M <= 64 of these shapes, its kernel with one pass over K
 * where that is faster (x and q exact in the products, fp32 accumulation; M <= 32 needs no workspace).  Other M > 1 runs on the fp16 matrix cores (the kernel of
 * qail_w4a16_linear for M > 16 with byte codes: K % 64 == 0, group_size % 64 == 0, an even
 * number of scales; (q * s) is rounded once to fp16 before the fp32 accumulation) and needs the
 * workspace the query below reports, 256-byte aligned.  Shapes outside both go to a plain
 * one-thread-per-output kernel.  Errors as for qail_w4a16_linear. */
int qail_w8a16_workspace(const qail_wdesc* d, int32_t M, size_t* bytes);
int qail_w8a16_linear(const qail_wdesc* d, const uint32_t* qweight, const uint16_t* scales,
                      const uint16_t* x, uint16_t* y, int32_t M, void* workspace,
                      size_t workspace_bytes, void* stream);

/* One linear of a batch for qail_w8a16_linear_batch (device pointers, 16-byte aligned). */
typedef struct {
    qail_wdesc d;
    const uint32_t* qweight;
    const uint16_t* scales;
    const uint16_t* x;   /* bf16 [M][K] */
    uint16_t* y;         /* bf16 [M][N] */
} qail_w8a16_item;

/* `count` independent 8-bit weight-only linears with the same M, given as a HOST array
 * (Sec. 5.4 also deploys the backbone with 8-bit weights: a decode step is again four such
 * linears per layer, a prefill pass four such GEMMs).  At M = 1 the items the streaming kernel
 * takes share launches (up to 8 each), every item on a share of the blocks, with the single
 * calls' results bit for bit; at M > 1 up to 8 consecutive items of the matrix-core path share
 * launches the same way (a different division of K than in a call of its own, so equal within
 * the W4A16 tolerance rather than bit for bit).  count >= 0 (0 is a no-op); workspace as
 * reported by the batch query; errors as for the single call. */
int qail_w8a16_batch_workspace(const qail_w8a16_item* items, int32_t count, int32_t M, size_t* bytes);
int qail_w8a16_linear_batch(const qail_w8a16_item* items, int32_t count, int32_t M, void* workspace,
                            size_t workspace_bytes, void* stream);

/* ------------------------------------------------------- training-side operators --
 * Sec. 4.1 / Algorithm 1: the quantised policy is trained through its quantisers with the
 * straight-through estimator.  Sec. 4.2 / Eq. 3: the QBC term; the appendix instantiates its
 * discrepancy as the mean L2 distance between the two policies' final logits. */

/* Forward of quantisation-aware training for a 4-bit group-quantised weight: w_hat =
 * dequantise(quantise(w)) with the ASYM_GROUP quantiser above, fp32 [N][K] -> fp32 [N][K]
 * (exact: (q - z) * s has at most 16 significant bits).  Its straight-through backward is the
 * identity, so no call exists for it. */
int qail_fake_quant_w4(const qail_wdesc* d, const float* w, float* w_hat, void* stream);

/* Learned-step quantiser (named in Sec. 5.1 for the driving policy): v_hat = clamp(rint(v / *s),
 * qn, qp) * *s in fp32; s: device, one float; qn <= 0 <= qp. */
int qail_lsq_forward(const float* v, size_t n, const float* s, int32_t qn, int32_t qp, float* v_hat,
                     void* stream);

/* Straight-through backward: dv = dout where qn <= v / s <= qp, else 0;
 * *ds = grad_scale * sum dout * t, t = rint(v/s) - v/s inside, qn below, qp above (fp32 sums in
 * a fixed order).  workspace: qail_lsq_backward_workspace bytes, 16-byte aligned. */
int qail_lsq_backward_workspace(size_t* bytes);
int qail_lsq_backward(const float* v, const float* dout, size_t n, const float* s, int32_t qn, int32_t qp,
                      float grad_scale, float* dv, float* ds, void* workspace, size_t workspace_bytes,
                      void* stream);

/* *loss = mean_b || logits_q[b] - logits_fp[b] ||_2 over fp32 [B][D]; grad_q (optional, [B][D]) =
 * d loss / d logits_q = (diff / ||diff||) / B, zero for rows with zero distance.
 * workspace: B floats, 16-byte aligned. */
int qail_qbc_loss(const float* logits_q, const float* logits_fp, int32_t B, int32_t D, float* loss,
                  float* grad_q, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------- serving: between a decoder's linears --
 * The appendix "Analysis" times the prefill and the decode stage of the whole backbone.  These calls are what
 * a decoder layer does between its quantised linears when several requests are served at once: norms, a cache of
 * keys and values in pages, attention over it, and adapters that differ from request to request. */

/* Root-mean-square norm of rows, with the residual's addition before it:
 *     h = x (+ residual)                             fp32, one rounding
 *     r[m] = 1 / sqrt(mean_k h[m][k]^2 + eps)        fp32 sums
 *     y[m][k] = bf16(h[m][k] * r[m] * weight[k])
 * and, for 8-bit linears, codes with one step per row:
 *     u = h * weight                                 fp32, one rounding
 *     s = max_k |u[m][k]| / 127                      fp32, correctly rounded; 1 for an all-zero row, NaN where a u is not finite
 *     q[m][k] = clamp(rint(u / s), -127, 127);       y_scale[m] = s * r[m]
 * so q * y_scale stands for y; r is in the scale alone and decides no code.  Codes are packed as by qail_quantize_act_s8:
 * a row is the a_s8 of a qail_w8a8_gemm with H = W = 1, whose int32 sums are scaled by y_scale[m] and the weight's scale.
 *   x, residual  bf16 [M][K] (residual may be NULL); weight bf16 [K]; eps > 0
 *   h_out        bf16 [M][K], the rounded h, or NULL; may be x or residual itself
 *   y            bf16 [M][K] or NULL; may be x or residual itself, when h_out is not
 *   y_s8, y_scale  uint32 [M][K/4] and fp32 [M], both or neither
 * At least one of h_out (with a residual), y and y_s8 is required.  K % 8 == 0, K <= 32768, M * K < 2^31, 1 <= M < 2^26. */
int qail_rmsnorm(const uint16_t* x, const uint16_t* residual, const uint16_t* weight, float eps, int32_t M, int32_t K,
                 uint16_t* h_out, uint16_t* y, uint32_t* y_s8, float* y_scale, void* stream);

/* Its gradient, at the rounded h: bf16 [M][K], h_out of the forward call, or x where there is no residual (the forward call with a residual normalises the
 * sum before its rounding to bf16; the two gradients differ by what that rounding changes);
 * dy: the gradient of y; dres: the gradient that reaches h_out on its other way, or NULL; both bf16 [M][K].  With n = h * r:
 *     dx = bf16(r * (dy * weight - n * mean_k(dy * weight * n)) + dres)     the gradient of x and of residual; [M][K]
 *     dweight[k] = sum_m dy * n                                             fp32 [K], a fixed order of summation
 * (for codes the straight-through gradient is that of y).  dx may be h, dy or dres itself.  The workspace is 16-byte aligned. */
int qail_rmsnorm_backward_workspace(int32_t M, int32_t K, size_t* bytes);
int qail_rmsnorm_backward(const uint16_t* h, const uint16_t* weight, float eps, const uint16_t* dy, const uint16_t* dres,
                          int32_t M, int32_t K, uint16_t* dx, float* dweight, void* workspace, size_t workspace_bytes,
                          void* stream);

/* How a cache holds keys and values. */
typedef enum {
    QAIL_KV_BF16 = 0,
    QAIL_KV_S8 = 1    /* signed codes -127..127 with one fp32 step per token and head: max|t| / 127, 1 for an all-zero row,
                         NaN where a value is not finite */
} qail_kv_type;

/* The keys and values of one layer in pages that requests are given as they grow.  k and v (and their steps) are
 * [num_pages][heads][page_size][head_dim] (steps without the last dimension); device memory, 16-byte aligned. */
typedef struct {
    void* k;
    void* v;
    float* k_scale;      /* QAIL_KV_S8 only */
    float* v_scale;
    int32_t num_pages, heads, page_size;   /* page_size: a power of two, 16 to 1024 */
    int32_t head_dim;                      /* 64 or 128 */
    int32_t type;                          /* qail_kv_type */
} qail_kv_cache;

/* Byte sizes of k (and of v), and of k_scale (and of v_scale); pointers in `c` are not looked at. */
int qail_kv_cache_sizes(const qail_kv_cache* c, size_t* data_bytes, size_t* scale_bytes);

/* The requests of a step.  Their new tokens are packed: request r has rows q_start[r] .. q_start[r + 1] - 1 of the step's tensors,
 * any number of them (0: it waits).  kv_len[r] counts its tokens with the new ones, so that row i of them has position
 * kv_len[r] - (q_start[r + 1] - q_start[r]) + i; a token at position p lies in slot p % page_size of page page_table[r][p / page_size].
 * page_table, q_start and kv_len are device memory (4-byte aligned), read when the kernels run, so that a captured graph can be
 * replayed with other contents: q_start ascends from 0 to `tokens`.
 * tokens < 2^24, requests <= 2^20, max_pages * page_size <= 2^30; for attention requests * heads of the cache <= 2^22 and tokens * q_heads <= 2^30.
 * max_new and max_len are upper bounds on a request's new tokens and its kv_len that the launches are planned by; contents
 * beyond them cost speed, not results. */
typedef struct {
    const int32_t* page_table;   /* [requests][max_pages]; entries that no token lies in are not used */
    const int32_t* q_start;      /* [requests + 1] */
    const int32_t* kv_len;       /* [requests] */
    int32_t requests, max_pages;
    int32_t tokens;              /* rows of the step's tensors, >= 0 */
    int32_t max_new, max_len;
} qail_requests;

/* `errors` (device, one uint32, may be NULL; not cleared) of the two calls below is incremented at least once if the contents of the
 * three arrays are bad: a page outside 0 .. num_pages - 1 for a token that the call reads or writes, a kv_len that is negative or beyond
 * max_pages * page_size (of a request that waits as well), a q_start that descends or leaves 0 .. tokens, for qail_kv_append a negative position
 * or one beyond `positions`.  Nothing outside the given buffers is read or written then; the outputs of the requests concerned are unspecified.
 * A step of zero tokens launches nothing and looks at nothing. */

/* Rotates the new tokens' keys and queries and writes keys and values to their slots.  With half = head_dim / 2, position p, i < half,
 * each product and sum one fp32 operation (no fused multiply-add):
 *     t'[i] = t[i] * cos[p][i] - t[i + half] * sin[p][i],   t'[i + half] = t[i + half] * cos[p][i] + t[i] * sin[p][i]
 * rounded once, to bf16 or to the cache's codes.
 *   k, v      bf16, token t and head h at t * k_stride + h * head_dim (elements; strides are multiples of 8, >= heads * head_dim)
 *   q, q_out  bf16, q_heads heads of each; q as k with q_stride, q_out contiguous [tokens][q_heads][head_dim] (may be q where that is
 *             contiguous); both NULL where there are no queries to rotate
 *   cos, sin  fp32 [positions][half], both or neither: without them nothing is rotated and q must be NULL
 * The pages that requests write to must differ. */
int qail_kv_append(const qail_kv_cache* c, const qail_requests* b, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                   int64_t v_stride, const uint16_t* q, int64_t q_stride, int32_t q_heads, uint16_t* q_out, const float* cos,
                   const float* sin, int32_t positions, uint32_t* errors, void* stream);

/* Causal attention of the new tokens over their requests' cache, which holds their own keys and values already:
 *     out[t][a] = sum_j p_j v[j],  p = softmax_j(scale * q[t][a] . k[j]),  j = 0 .. position of t, head a / (q_heads / heads) of the cache
 * (q_heads is a multiple of the cache's heads).  A chunk may be one token, a few, or a whole prompt.  Scores, maxima and sums are fp32.  For its
 * product with v, p is held to 2^-16 of it where a request has at most 16 rows (new tokens times q_heads / heads) and rounded to bf16 where it has
 * more; one that is below 2^-126 of its row's largest may count as zero.  A token whose position is negative (more new tokens than kv_len) sees no key: its
 * rows are zero; one whose scores are all minus infinity is NaN.  The sum of p_j v[j] is formed before it is divided by the sum of p, and overflows
 * where it passes fp32's range.  Slots behind a request's last token may hold anything; what a token does not see, infinities and NaN of later tokens
 * included, does not reach its rows.
 *   q         bf16, token t and head a at t * q_stride + a * head_dim; q_stride % 8 == 0
 *   out       bf16 [tokens][q_heads][head_dim]
 *   scale     > 0, finite
 * The workspace (256-byte aligned; may be NULL where the query says 0) holds the partial results of keys that are divided among blocks. */
int qail_paged_attention_workspace(const qail_kv_cache* c, const qail_requests* b, int32_t q_heads, size_t* bytes);
int qail_paged_attention(const qail_kv_cache* c, const qail_requests* b, const uint16_t* q, int64_t q_stride, int32_t q_heads, float scale,
                         uint16_t* out, uint32_t* errors, void* workspace, size_t workspace_bytes, void* stream);

/* Low-rank adapters of many requests beside a shared 4-bit linear: `count` linears as for qail_w4a16_linear_batch, and for each a stack
 * of `n` adapters of one rank, of which row m of x uses row_adapter[m]:
 *     y[m] = x[m] w_hat^T + scaling[a] (x[m] A[a]^T) B[a]^T,  a = row_adapter[m];  without the second term where a is not in 0 .. n - 1
 * A: bf16 [n][r][K], B: bf16 [n][N][r], scaling: fp32 [n]; device memory, 16-byte aligned; 8 <= r <= 64, r % 8 == 0, n >= 1; an
 * adapter of a lower rank is filled up with zeros.  row_adapter: int32 [M], device, 4-byte aligned, the same for all linears.
 * The linear is rounded to bf16 as by qail_w4a16_linear_batch, the adapter's fp32 part is added and rounded again; a row without an adapter
 * keeps the linear's bits.  What one adapter holds reaches no row of another.  M >= 1: a step of zero tokens, which the writer and the attention take,
 * has nothing to multiply, here and in the norm as in every linear. */
typedef struct {
    const uint16_t* A;
    const uint16_t* B;
    const float* scaling;
    int32_t n, r;
} qail_adapters;

/* Workspace (256-byte aligned): the linears' own and the down-projections x A^T in fp32.  Errors as for qail_w4a16_linear_lora_batch. */
int qail_w4a16_adapters_workspace(const qail_w4a16_item* items, const qail_adapters* adapters, int32_t count, int32_t M, size_t* bytes);
int qail_w4a16_linear_adapters_batch(const qail_w4a16_item* items, const qail_adapters* adapters, const int32_t* row_adapter, int32_t count,
                                     int32_t M, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------- the policy's ends, in 16 bits --
 * Sec. 5.4 and the appendix "Analysis" quantise the backbone's linears; the table of embeddings, the head, the projector and the vision
 * side stay in 16 bits.  These calls are what a policy does before its first decoder layer and after its last one.  Their workspaces carry
 * nothing between calls; calls that share one must be ordered on one stream. */

/* Rows of a table: h[t][k] = bf16(scale * table[ids[t]][k]), one rounding.
 *   table  bf16 [V][K]; ids int32 [T]; h bf16 [T][K] (not the table); scale finite
 * A row whose id is negative is left as it was: image patches, written by the projector, lie between the tokens.  For an id >= V the row
 * is zero and *errors (device, one uint32, may be NULL; not cleared) is incremented at least once.
 * K % 8 == 0, K <= 65536, V < 2^24, 0 <= T < 2^24 (0 launches nothing), V * K and T * K <= 2^36. */
int qail_embed(const uint16_t* table, int32_t V, int32_t K, const int32_t* ids, int32_t T, float scale, uint16_t* h, uint32_t* errors,
               void* stream);

/* Its gradient: dtable[v][k] = scale * sum of dh[t][k] over the t with ids[t] == v, fp32 [V][K], in an order that depends on ids alone, so
 * that the same call always gives the same bits; accumulate != 0 adds it to what dtable holds and leaves the rows without a token alone,
 * 0 overwrites all of it.  Negative ids and ids >= V have no row; the latter are counted as above.  What dh holds in their rows is not used.
 * dtable is neither dh nor ids.  Sizes as above, T = 0 among them (with accumulate == 0 the gradient is zero).  The workspace is 256-byte aligned. */
int qail_embed_backward_workspace(int32_t V, int32_t K, int32_t T, size_t* bytes);
int qail_embed_backward(const int32_t* ids, const uint16_t* dh, int32_t T, float scale, int32_t V, int32_t K, int32_t accumulate, float* dtable,
                        uint32_t* errors, void* workspace, size_t workspace_bytes, void* stream);

typedef enum {
    QAIL_ACT_NONE = 0,
    QAIL_ACT_RELU = 1,       /* max(z, 0); slope 0 at 0 */
    QAIL_ACT_GELU = 2,       /* z (1 + erf(z / sqrt(2))) / 2 */
    QAIL_ACT_GELU_TANH = 3,  /* z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2 */
    QAIL_ACT_SILU = 4        /* z / (1 + exp(-z)) */
} qail_activation;

/* A linear whose weights stay in 16 bits: W bf16 [N][K], bias bf16 [N] or NULL; device memory, 16-byte aligned. */
typedef struct {
    int32_t N, K;             /* N >= 1; K >= 8, a multiple of 8 */
    int32_t activation;       /* qail_activation */
    const uint16_t* weight;
    const uint16_t* bias;
    int32_t round_dz;         /* of the gradients, below: 0 or not */
} qail_w16a16;

/*     z[m][n] = sum_k x[m][k] W[n][k] + bias[n]           fp32
 *     y[m][n] = act(z[m][n]) + residual[m][n]              fp32, rounded once
 *   x          bf16 [M][K]; residual bf16 [M][N] or NULL
 *   y, y_f32   bf16 or fp32 [M][N], exactly one of them; y may be the residual itself
 *   z_out      bf16 [M][N], the rounded z for the backward call, or NULL
 * No output may be an input otherwise, or another output.  M >= 1; M, N, K <= 2^22, M * N, M * K and N * K <= 2^33.  The workspace (256-byte
 * aligned; may be NULL where the query says 0) holds partial sums of output tiles whose K is divided among blocks. */
int qail_w16a16_workspace(const qail_w16a16* d, int32_t M, size_t* bytes);
int qail_w16a16_linear(const qail_w16a16* d, const uint16_t* x, int32_t M, const uint16_t* residual, uint16_t* z_out, uint16_t* y, float* y_f32,
                       void* workspace, size_t workspace_bytes, void* stream);

/* Its gradients, at the rounded z:
 *     dz = dy * act'(z)                     fp32; enters the products in two bf16 parts (2^-16 of itself), or with round_dz != 0 rounded to
 *                                           bf16, which takes 0.54 to 0.65 of the call's time and costs the gradients as much as their own rounding;
 *                                           a bf16 dy without an activation or with RELU is exact either way
 *     dx[m][k] = sum_n dz[m][n] W[n][k]     fp32 sums, rounded once; bf16 [M][K] or NULL
 *     dweight[n][k] = sum_m dz[m][n] x[m][k]   likewise; bf16 [N][K] or NULL
 *     dbias[n] = sum_m dz[m][n]             of the unrounded dz, a fixed order of summation; fp32 [N] or NULL
 * (that of the residual is dy).
 *   x            needed for dweight only
 *   z            z_out of the forward call, bf16 [M][N]; not looked at without an activation
 *   dy, dy_f32   bf16 or fp32 [M][N], exactly one of them
 * At least one of the three outputs is required, and each is written whole; none may be an input.  Sizes as above. */
int qail_w16a16_backward_workspace(const qail_w16a16* d, int32_t M, size_t* bytes);
int qail_w16a16_backward(const qail_w16a16* d, const uint16_t* x, const uint16_t* z, const uint16_t* dy, const float* dy_f32, int32_t M,
                         uint16_t* dx, uint16_t* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* stream);

typedef enum { QAIL_LOGITS_BF16 = 0, QAIL_LOGITS_F32 = 1 } qail_logits_type;

/* How the rows of a step are drawn from: one value a row, device memory, 4-byte aligned; a NULL array leaves its choice off in all rows. */
typedef struct {
    const float* temperature;   /* > 0; 0: the largest logit.  Off: 1 */
    const int32_t* top_k;       /* <= 0: off */
    const float* top_p;         /* >= 1: off; <= 0 keeps the first token alone */
    const float* min_p;         /* <= 0: off */
} qail_sampling;

/* A token for each row of logits [R][V], row r at r * stride (elements, >= V).  With the tokens of a row in the order of falling logits, equal
 * ones in the order of their numbers, w[j] = exp((logit[j] - the row's largest) / temperature):
 *     top_k keeps the first top_k tokens of that order; top_p, of what is kept, the shortest leading part whose sum of w is at least
 *     top_p of the sum of all that is kept; min_p, of those, the ones with w >= min_p; the first token is always kept
 *     token[r] = the lowest j that is kept with sum_{i <= j, i kept} w[i] > u[r] * sum_{i kept} w[i]
 *     logprob[r] = log(w[token] / sum_{i kept} w[i]), fp32; 0 at temperature 0
 * w and its sums are held in 64 bits, as multiples of 2^-44: a token below 2^-45 of its row's largest counts as impossible, and the order of
 * the sums does not matter, so that the same call always gives the same tokens.
 *   logits   of `type`, 16-byte aligned; minus infinity: never drawn
 *   u        fp32 [R], in [0, 1): the random numbers; not looked at where temperature is 0
 *   token    int32 [R]; logprob fp32 [R] or NULL
 * A row that holds NaN or plus infinity or nothing above minus infinity, whose temperature is negative, infinite or NaN, whose top_p or min_p is NaN or whose u is outside
 * [0, 1) gets token -1 and logprob NaN, and *errors (device, one uint32, may be NULL; not cleared) is incremented.
 * 0 <= R <= 2^20, 1 <= V <= 2^18. */
int qail_sample(const void* logits, int32_t type, int64_t stride, int32_t R, int32_t V, const qail_sampling* s, const float* u, int32_t* token,
                float* logprob, uint32_t* errors, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* QAIL_H */
