/*
 * linfusion_block.h — C ABI of the operators that stand before and after the attention of
 * linfusion_attn.h inside a transformer block: rotary positions with several axes on Q and K, and
 * the norms before and after a block fused with its modulation, gate and residual scale.  Each has
 * its backward pass.  Same library, status codes and conventions as linfusion_attn.h:
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
 * a multiple of 8 (that of an axis of one is not looked at).  Arithmetic, row statistics and sums are
 * fp32; each 16-bit output is rounded once, to nearest even.
 */
#ifndef LINFUSION_BLOCK_H
#define LINFUSION_BLOCK_H

#include "linfusion_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------------------
 * Rotary positions with several axes (time, height, width, ...).
 *
 * Of a head's d channels the first 2 * P are rotated, P = pairs[0] + ... + pairs[n_axes - 1]; the
 * others are copied.  Pair p belongs to the axis whose share it falls in; as the i-th of the n pairs
 * of axis a it is turned, for a token at position pos[a], by the angle
 *
 *     angle = pos[a] * theta^(-i / n)
 *     (u, w) -> (u cos - w sin,  u sin + w cos)          backward: the angle's negative
 *
 * where (u, w) are channels (2p, 2p + 1) when `interleaved` is set, else (p, p + P).  The rotation is
 * orthogonal, so the backward pass (gradients of the rotated tensor in, of the unrotated one out) is
 * the rotation by the negative angle.
 * ---------------------------------------------------------------------------------------------- */
#define LINFUSION_ROPE_MAX_AXES 4
#define LINFUSION_ROPE_MAX_WIDTH 256
typedef struct {
    int32_t B;                               /* batch, 1 .. 65535                             */
    int32_t N;                               /* tokens, >= 1                                  */
    int32_t d;                               /* head width, a multiple of 8, <= 256           */
    int32_t n_axes;                          /* 1 .. 4                                        */
    int32_t pairs[LINFUSION_ROPE_MAX_AXES];  /* pairs of each axis, >= 0; 2 <= 2 * sum <= d   */
    int32_t interleaved;                     /* pairs (2p, 2p + 1) (1) or (p, p + P) (0)      */
    int32_t backward;                        /* rotate by the negative angle                  */
    double theta;                            /* finite, > 0; below 1 frequencies pass 1       */
    uint32_t flags;                          /* 0 or LINFUSION_DTYPE_FP16                     */
} linfusion_rope_desc_t;

/* One tensor of B x N x heads rows; `out` may be `in` itself with the same strides (in place) and must
 * not overlap it otherwise, nor the other tensor (Q and K may be interlaced views of one tensor: then with the
 * same batch and token strides).  heads = 0: the tensor is absent. */
typedef struct {
    const void* in;
    void* out;
    int32_t heads;
    int64_t in_batch, in_token, in_head;     /* element strides, multiples of 8, >= 0 (in: 0 broadcasts) */
    int64_t out_batch, out_token, out_head;  /* element strides, multiples of 8, >= 0 */
} linfusion_rope_tensor_t;

/*
 * Rotate Q and K (either may be absent) in one launch.  positions: fp32 device memory, the n_axes
 * coordinates of token n of batch b at positions + b * pos_batch_stride + n * n_axes;
 * pos_batch_stride 0 shares them over the batch.  Coordinates need not be whole (interpolated
 * positions).  The angle is formed from a frequency held in two fp32 parts and reduced to one turn
 * before the sine and cosine, so it is good to about 3e-7 for angles below 2^24 radians (coordinates below 2^24 where
 * theta >= 1), and to 2^-46 of the angle beyond.
 * Errors: INVALID_ARG (null / misaligned pointers, bad sizes or strides, both tensors absent, a theta so small that a
 * frequency passes 1e30),
 * UNSUPPORTED (unknown flags, d > 256), CUDA.
 */
linfusion_status_t linfusion_rope(const linfusion_rope_desc_t* desc, const linfusion_rope_tensor_t* q,
                                  const linfusion_rope_tensor_t* k, const float* positions,
                                  int64_t pos_batch_stride, void* cuda_stream);

/* ------------------------------------------------------------------------------------------------
 * The norms before and after a block.  x is the residual stream, a the output of the block behind it,
 * both [B, N, C]; the vectors are per channel, gate / scale / shift of each batch entry or shared.
 *
 *     y = residual_scale * x + gate * (Post(a) * post_weight + post_bias)      where a is given, else y = x
 *     n = (Pre(y) * pre_weight + pre_bias) * (1 + scale) + shift                 the next block's input
 *
 * Post and Pre are each absent (the identity; n is then not computed), a layer norm
 * (v - mean) / sqrt(var + eps) or an RMS norm v / sqrt(mean(v^2) + eps) over the C channels, with the
 * variance taken about the mean (two steps, nothing cancels).  Absent vectors count as gate = 1, weight
 * = 1, bias = 0, scale = 0, shift = 0.  Pre reads y as it is stored (rounded to 16 bits), so that the
 * backward pass, which is given y, differentiates what ran.
 * ---------------------------------------------------------------------------------------------- */
typedef enum { LINFUSION_NORM_NONE = 0, LINFUSION_NORM_LAYER = 1, LINFUSION_NORM_RMS = 2 } linfusion_norm_t;
#define LINFUSION_BLOCK_NORM_MAX_C 8192
typedef struct {
    int32_t B;             /* 1 .. 65534                                   */
    int32_t N;             /* rows of a batch entry, >= 1                  */
    int32_t C;             /* channels, a multiple of 8, <= 8192           */
    int32_t pre, post;     /* linfusion_norm_t                             */
    float eps;             /* finite, >= 0                                 */
    float residual_scale;  /* finite                                       */
    uint32_t flags;        /* 0 or LINFUSION_DTYPE_FP16                    */
} linfusion_block_norm_desc_t;

/* A [B, N, C] tensor: element strides of the batch and of a row, multiples of 8, >= 0. */
typedef struct {
    void* p;
    int64_t batch, row;
} linfusion_rows_t;
/* Per-channel vector: entry b at p + b * batch; batch = 0 shares one vector over the batch.  p NULL: absent. */
typedef struct {
    const void* p;
    int64_t batch;
} linfusion_channels_t;

typedef struct {
    linfusion_channels_t gate, scale, shift;                       /* scale and shift come together */
    const void *pre_weight, *pre_bias, *post_weight, *post_bias;   /* [C]; need their norm           */
} linfusion_block_norm_vectors_t;

/*
 * One launch.  x and a are read; y (with a; may be x or a in place) and n (with pre) are written.  Otherwise the
 * address range of an output (first to last byte) must not meet that of an input or of the other output.  Without a, y must be NULL and post NONE, gate absent.
 * Errors: INVALID_ARG, UNSUPPORTED (C > 8192 or not a multiple of 8, unknown flags or norms), CUDA.
 */
linfusion_status_t linfusion_block_norm(const linfusion_block_norm_desc_t* desc, const linfusion_rows_t* x,
                                        const linfusion_rows_t* a, const linfusion_block_norm_vectors_t* v,
                                        const linfusion_rows_t* y, const linfusion_rows_t* n, void* cuda_stream);

/* Gradients of the vectors, fp32, NULL where not wanted: [C], summed over the batch, or, of a gate, scale or shift that has a
 * batch stride or its bit in `per_entry`, dense [B, C].  (The bit is for one vector seen by every entry through a stride of 0
 * whose gradients are wanted entry by entry.) */
#define LINFUSION_PER_ENTRY_GATE 1u
#define LINFUSION_PER_ENTRY_SCALE 2u
#define LINFUSION_PER_ENTRY_SHIFT 4u
typedef struct {
    float *gate, *scale, *shift, *pre_weight, *pre_bias, *post_weight, *post_bias;
    uint32_t per_entry;
} linfusion_block_norm_grads_t;

/*
 * Backward.  y: the stream as the forward pass stored it (x where there is no a; not read without pre).
 * dy: the gradient of y from everything but n (NULL: zero); dn: the gradient of n (with pre).
 * dx = residual_scale * (dy + gradient through Pre) (without a: no residual_scale), and with a the gradient da.  Row statistics are
 * computed again from y and a, so the forward pass keeps nothing.  dx may lie exactly over dy and da exactly over a, with the
 * same strides; otherwise the address range of an output, a gradient of a vector among them, must not meet that of an input or of
 * another output, nor the workspace any of them.
 * workspace: device memory, 256-byte aligned, of linfusion_block_norm_workspace_bytes(); used until the
 * call's kernels have run, and may then be used by anything else.
 * Two launches (one where no gradient of a vector is wanted).  Errors: as above, ALLOC (workspace too small).
 */
linfusion_status_t linfusion_block_norm_backward(const linfusion_block_norm_desc_t* desc, const linfusion_rows_t* y,
                                                 const linfusion_rows_t* a, const linfusion_block_norm_vectors_t* v,
                                                 const linfusion_rows_t* dy, const linfusion_rows_t* dn,
                                                 const linfusion_rows_t* dx, const linfusion_rows_t* da,
                                                 const linfusion_block_norm_grads_t* grads, void* workspace,
                                                 size_t workspace_bytes, void* cuda_stream);
/* Pure host computation; `sm_count` <= 0 means 148.  Never less than the call needs on a device with that many SMs. */
linfusion_status_t linfusion_block_norm_workspace_bytes(const linfusion_block_norm_desc_t* desc, int32_t sm_count,
                                                        size_t* bytes);

#ifdef __cplusplus
}
#endif
#endif
