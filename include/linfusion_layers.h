/*
 * linfusion_layers.h — C ABI of a block's own layers, beside the attention of linfusion_attn.h and the
 * operators around it in linfusion_block.h: matrix products with bias, activation and residual in
 * their epilogue, a gated linear recurrence over the tokens (of the kind that Eq. 3 of the paper gates, but each
 * channel for itself: a state of one value, no B and no C), and activation checkpoints in 8 bits that both backward passes read.
 * Same library, status codes and conventions as linfusion_block.h:
 *
 * Every function returns a status code; nothing throws or aborts across this boundary.  Calls only
 * enqueue work on the given stream (a cudaStream_t; NULL is the legacy default stream) of the
 * CURRENT device, which must be the one the tensors live on; they allocate nothing and keep no
 * state, so calls on different streams or threads are independent as long as their outputs and
 * workspaces are.  Results are bit-identical from call to call for identical inputs on the same
 * device (fixed summation order, no floating-point atomics).  All of them can be captured into a
 * CUDA graph.
 *
 * Tensors are 16-bit (bf16, or fp16 with LINFUSION_DTYPE_FP16) device memory.  Strides count
 * elements; the channels of a row are contiguous.  Every pointer is 16-byte aligned and every stride
 * a multiple of 8 (that of an axis of one is not looked at).  Arithmetic and sums are fp32; each
 * 16-bit output is rounded once, to nearest even.
 */
#ifndef LINFUSION_LAYERS_H
#define LINFUSION_LAYERS_H

#include "linfusion_block.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------------------
 * Checkpoints in 8 bits.  32 consecutive channels of a row (the last group of a row may be shorter)
 * share a power of two:
 *
 *     e    = the smallest whole number with max|x| <= 127 * 2^e, held to -126 .. 121 (bf16) or -24 .. 9 (fp16)
 *     code = x * 2^-e rounded to the nearest whole number (ties to even), held to -127 .. 127
 *
 * codes: int8 [rows, C]; scales: uint8 [rows, ceil(C / 32)], the byte e + 127; both dense.  A value is off by at most
 * max|x| / 127 of its group (half a step; one at the top of the range), or by 2^-127 where that is more (bf16).  An fp32 value beyond the
 * range (a pre-activation above 65024 in fp16) is kept as 127 of the largest steps.  Because the scale is a power of two, code * 2^e has at most seven
 * significant bits and is a number of the storage type: reading a checkpoint rounds nothing, so a product on
 * 16-bit operands may read one as it is.  A value that is not finite has the code -128 and reads as NaN (the
 * recurrence's decay: as -infinity); the maximum is that of the finite ones.
 * ---------------------------------------------------------------------------------------------- */
#define LINFUSION_PACK8_GROUP 32
typedef struct {
    int32_t B;       /* batch, >= 1                       */
    int32_t N;       /* rows of a batch entry, >= 1       */
    int32_t C;       /* channels, a multiple of 8, >= 8   */
    uint32_t flags;  /* 0 or LINFUSION_DTYPE_FP16         */
} linfusion_pack8_desc_t;

/* A [B, N, C] tensor in 8 bits: rows b * N + n, both dense; codes 16-byte aligned. */
typedef struct {
    void* codes;
    void* scales;
} linfusion_packed8_t;

/* x -> packed, and back.  The address ranges of input and outputs must not meet.  Errors: INVALID_ARG, UNSUPPORTED (unknown
 * flags, 2^31 groups or more), CUDA. */
linfusion_status_t linfusion_pack8(const linfusion_pack8_desc_t* desc, const linfusion_rows_t* x, const linfusion_packed8_t* packed,
                                   void* cuda_stream);
linfusion_status_t linfusion_unpack8(const linfusion_pack8_desc_t* desc, const linfusion_packed8_t* packed, const linfusion_rows_t* x,
                                     void* cuda_stream);

/* ------------------------------------------------------------------------------------------------
 * A gated linear recurrence, each channel for itself.  Over the tokens in order (or from the last to the first):
 *
 *     L_t = rate * sigmoid(decay_t)       e_t = 1 - exp(-L_t)        v_t = sigmoid(gate_t) * x_t   (x_t without a gate)
 *     h_t = h_(t-1) + e_t (v_t - h_(t-1)) = exp(-L_t) h_(t-1) + (1 - exp(-L_t)) v_t,     h_(-1) = h0 (zero without one)
 *
 * x, decay, gate, h [B, N, C]; rate fp32 [C], >= 0 (a negative one counts as NaN, an infinite one as fp32's largest number); h0, last fp32 [B, C].  A token with decay = -infinity leaves the state
 * as it is, whatever its x and gate hold (NaN too): padding.  In a checkpoint of decay the code -128 counts as -infinity, so that padding
 * goes through one; a decay of +infinity or NaN cannot be told from it any more (from 17 on the sigmoid is 1: a finite decay does for
 * +infinity).  `state` keeps the states before every 64th token of
 * the scan, fp32 [B, ceil(N / 64), C]; the backward pass recomputes h from them, 64 tokens at a time, and needs no h.
 *
 * Backward, G_t the gradient of everything that follows from h_t (dlast, the gradient of the last state, with it):
 *
 *     G_t = dh_t + exp(-L_(t+1)) G_(t+1)        dv = e G        dL = exp(-L) (v - h_(t-1)) G
 *     dx = sigmoid(gate) dv      dgate = sigmoid'(gate) x dv    ddecay = rate sigmoid'(decay) dL
 *     drate = sum over batch and tokens of sigmoid(decay) dL    dh0 = exp(-L_0) G_0
 * ---------------------------------------------------------------------------------------------- */
#define LINFUSION_RECURRENCE_EVERY 64
typedef struct {
    int32_t B;        /* batch, 1 .. 65535                        */
    int32_t N;        /* tokens, >= 1                             */
    int32_t C;        /* channels, a multiple of 8, >= 8          */
    int32_t reverse;  /* 1: from the last token to the first      */
    uint32_t flags;   /* 0 or LINFUSION_DTYPE_FP16                */
} linfusion_recurrence_desc_t;

/* The inputs: `rows` of 16 bits, or, where packed.codes is given, a checkpoint (then of all inputs).  gate may be absent
 * (NULL, or neither given). */
typedef struct {
    linfusion_rows_t rows;
    linfusion_packed8_t packed;
} linfusion_recurrence_input_t;

/*
 * Forward, from 16-bit inputs.  Outputs: h (may lie exactly over x, decay or gate), and where given last and state (last may be
 * h0).  Otherwise the address range of an output must not meet that of an input or another output.
 * workspace: device memory, 256-byte aligned, of linfusion_recurrence_workspace_bytes(); used until the call's kernels
 * have run, and may then be used by anything else.  Up to 64 tokens: one launch and no workspace; else three launches.
 * Errors: INVALID_ARG, UNSUPPORTED (unknown flags, packed inputs, B above 65535, 2^31 tiles of 64 x 64 or more), ALLOC (workspace too
 * small), CUDA.
 */
linfusion_status_t linfusion_recurrence(const linfusion_recurrence_desc_t* desc, const linfusion_recurrence_input_t* x,
                                        const linfusion_recurrence_input_t* decay, const linfusion_recurrence_input_t* gate,
                                        const float* rate, const float* h0, const linfusion_rows_t* h, float* last, float* state,
                                        void* workspace, size_t workspace_bytes, void* cuda_stream);

typedef struct {
    linfusion_rows_t x, decay, gate; /* gate where there is one */
    float *rate, *h0;                /* fp32 [C], [B, C]; NULL where not wanted */
} linfusion_recurrence_grads_t;

/*
 * Backward.  state: as the forward pass kept it, else NULL: recomputed from the inputs and h0, into the workspace.  dlast: the
 * gradient of `last`, NULL: zero.  dx, ddecay and dgate may lie exactly over dh, or over their 16-bit inputs; otherwise the address
 * range of an output must not meet that of an input or another output, nor the workspace any of them.
 */
linfusion_status_t linfusion_recurrence_backward(const linfusion_recurrence_desc_t* desc, const linfusion_recurrence_input_t* x,
                                                 const linfusion_recurrence_input_t* decay, const linfusion_recurrence_input_t* gate,
                                                 const float* rate, const float* h0, const float* state, const linfusion_rows_t* dh,
                                                 const float* dlast, const linfusion_recurrence_grads_t* grads, void* workspace,
                                                 size_t workspace_bytes, void* cuda_stream);
/* Pure host computation: of a forward pass (backward = 0), a backward pass with saved states (1), one without (2). */
linfusion_status_t linfusion_recurrence_workspace_bytes(const linfusion_recurrence_desc_t* desc, int32_t backward, size_t* bytes);

/* ------------------------------------------------------------------------------------------------
 * A matrix product with its epilogue:
 *
 *     u = x w + bias          y = act(u) + residual
 *
 * x [M, K], y, residual, u [M, N]; w [K, N] with either axis contiguous (w_transposed: w[k, n] at w + n * w_stride + k, else at
 * w + k * w_stride + n); bias [N] of the storage type.  bias and residual may be absent.  u, the pre-activation that the
 * backward pass needs, is kept where asked for: in 16 bits, or as a checkpoint in 8 bits, straight from the fp32 sums.
 *
 * Backward:  du = dy * act'(u)      dx = du w^T      dw = x^T du      dbias = sum of du over the rows (fp32)
 *
 * du is rounded to 16 bits before the two products (they run on 16-bit operands); dbias sums it unrounded.  The gradient of the residual is dy.
 * The activations are good to 2e-5 of themselves before their rounding (1e-6 near zero), their slopes to as much of the terms that they are
 * the sum of.
 * ---------------------------------------------------------------------------------------------- */
typedef enum {
    LINFUSION_ACT_NONE = 0,
    LINFUSION_ACT_RELU = 1,
    LINFUSION_ACT_SILU = 2,
    LINFUSION_ACT_GELU = 3,      /* u Phi(u), Phi the normal distribution                  */
    LINFUSION_ACT_GELU_TANH = 4  /* u / 2 (1 + tanh(sqrt(2 / pi) (u + 0.044715 u^3)))     */
} linfusion_act_t;

typedef struct {
    int32_t M;             /* rows, >= 1                          */
    int32_t K;             /* input channels, a multiple of 8     */
    int32_t N;             /* output channels, a multiple of 8    */
    int32_t act;           /* linfusion_act_t                     */
    int32_t w_transposed;  /* 1: w is stored [N, K]               */
    uint32_t flags;        /* 0 or LINFUSION_DTYPE_FP16           */
} linfusion_linear_desc_t;

/* A [rows, channels] tensor: element stride of a row, a multiple of 8 and at least the channels, of inputs too (not looked at of a single row). */
typedef struct {
    void* p;
    int64_t row;
} linfusion_matrix_t;

/*
 * One launch.  y may lie exactly over residual.  Otherwise the address range of an output must not meet that of an
 * input or another output.  workspace: device memory, 256-byte aligned, of linfusion_linear_workspace_bytes() (0 for
 * many sizes; NULL is fine then); used until the call's kernel has run, and may then be used by anything else.
 * Errors: INVALID_ARG, UNSUPPORTED (K or N no multiple of 8, unknown flags or act), ALLOC (workspace too small), CUDA.
 */
linfusion_status_t linfusion_linear(const linfusion_linear_desc_t* desc, const linfusion_matrix_t* x, const linfusion_matrix_t* w,
                                    const void* bias, const linfusion_matrix_t* residual, const linfusion_matrix_t* y,
                                    const linfusion_matrix_t* u, const linfusion_packed8_t* u_packed, void* workspace,
                                    size_t workspace_bytes, void* cuda_stream);

/* What the backward pass reads besides dy and w: x and u each in 16 bits or as a checkpoint (of M rows). */
typedef struct {
    linfusion_matrix_t x, u;
    linfusion_packed8_t x_packed, u_packed;
} linfusion_linear_saved_t;

/*
 * dx [M, K], dw laid out as w is (its own stride, the same w_transposed), dbias fp32 [N]; each absent where not wanted.  u is not read
 * without an activation, x not without dw, w not without dx.
 * workspace: device memory, 256-byte aligned, of linfusion_linear_workspace_bytes(); used until the call's kernels have
 * run, and may then be used by anything else.  The address range of an output or of the workspace must not meet that of an input or another output.
 */
linfusion_status_t linfusion_linear_backward(const linfusion_linear_desc_t* desc, const linfusion_matrix_t* dy,
                                             const linfusion_linear_saved_t* saved, const linfusion_matrix_t* w,
                                             const linfusion_matrix_t* dx, const linfusion_matrix_t* dw, float* dbias,
                                             void* workspace, size_t workspace_bytes, void* cuda_stream);
/* Pure host computation: of a forward pass (backward = 0), of a backward pass with x in 16 bits (1), with x as a checkpoint
 * (2).  `sm_count` <= 0 means 148.  Never less than the call needs on a device with that many SMs. */
linfusion_status_t linfusion_linear_workspace_bytes(const linfusion_linear_desc_t* desc, int32_t backward, int32_t sm_count, size_t* bytes);

/* How many waits of this header's kernels expired on `device` since the library was loaded (0 in health; outputs of a call whose
 * wait expired are not to be used).  Synchronizes the stream. */
linfusion_status_t linfusion_layers_expired(int32_t device, uint32_t* count, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif
