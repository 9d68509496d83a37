/*
 * ssd_layers.h - C ABI of the layer operators next to the SSD-SGD update path: what makes a
 * worker's gradient, and what conditions it before ssd_step reads it (one NVIDIA B200, sm_100a).
 *
 *   ssd_linear_forward / _backward   y = act(x W^T + b) + r and its gradients
 *   ssd_gated_forward  / _backward   h = act(x Wg^T + bg) * (x Wu^T + bu) and its gradients
 *   ssd_clip_grad_norm               gradient norms over groups of tensors, and clipping
 *
 * Weight and bias gradients are written where the caller says, normally the tensors of a worker's
 * gradient arena (see ssd_tensor_offset), in either gradient type of the update path.
 *
 * Conventions (those of ssd_sgd.h where not said otherwise)
 *  - Matrices are row-major; `ld...` is the distance between two rows in ELEMENTS (at least the row's
 *    length; any value does when there is one row).  Pointers need the alignment of their element
 *    type only.  Rows whose start and pitch are multiples of 16 bytes are read in place; others are
 *    copied into the workspace first.
 *  - All memory is the caller's DEVICE memory, the workspace included; nothing is allocated or kept.
 *    The content of the workspace means nothing between calls; calls that can overlap on the GPU need
 *    one each.
 *  - Calls enqueue on `cuda_stream` and return.  Arguments are checked before anything is enqueued.  They can be made while the stream is
 *    captured into a graph, after a first call of the same kind outside one (which sets up the kernels on the device).
 *    An output overlaps no input, no other output and not the workspace (SSD_ERR_ARG).  Two matrices with equal
 *    row pitch whose columns lie side by side do not overlap.  One exception: `residual` and `y` may be the same matrix.
 *  - Numerics.  Products are summed in float32.  bfloat16 operands enter the tensor cores as they are.
 *    float32 operands enter as three bfloat16 parts of 8 bits each, which hold all 24 bits
 *    (down to steps of 2^-133, bfloat16's smallest: operands below 2^-109 have fewer); of their nine
 *    partial products the six largest are kept, which leaves out less than 2^-22 of |a b| (2^-26 on average), or the three
 *    largest where a weight gradient is rounded to bfloat16.  Calls of a few rows, or of little work, take no parts: float32
 *    multiply-adds, or the tensor cores on bfloat16 as it is.  The tensor cores cut where they add: sums for float32 results are
 *    therefore rounded to nearest every 512 products; those for bfloat16 results are not, the cuts being below their rounding.
 *    dz = dy * act'(z) is computed in float32 and rounded once to bfloat16 for bfloat16 results, or carried in
 *    three parts (in calls of a few rows: in float32) for float32 results.  Epilogues are computed in float32 and rounded
 *    once; gelu's Phi and silu's logistic function to an absolute 1e-6, so that far in their tails few digits are right.  Results do not depend on timing: the same call gives
 *    the same bits.  Which kernel takes a call, and so the order of its sums, depends on its sizes and alignment.
 *    A NaN or infinity in a row of x, or of a weight, reaches the outputs that depend on it (as NaN where float32
 *    operands are split) and no others.
 */
#ifndef SSD_LAYERS_H
#define SSD_LAYERS_H

#include "ssd_sgd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* relu(v) = max(v, 0); gelu(v) = v * Phi(v) with the normal distribution function Phi (erf form);
 * silu(v) = v / (1 + exp(-v)).  relu'(0) = 0. */
typedef enum { SSD_ACT_NONE = 0, SSD_ACT_RELU = 1, SSD_ACT_GELU = 2, SSD_ACT_SILU = 3 } ssd_act;

/* Linear layer, forward:  z = x W^T + bias,  y = act(z) + residual.
 * x [rows, in], weight [out, in], residual, y, z [rows, out] of type `dtype`; bias [out] float32.
 * bias, residual and z may be NULL (z: the pre-activation, which the backward pass needs unless
 * act is SSD_ACT_NONE).  rows >= 0, features >= 1, each below 2^31 - 2^16. */
typedef struct {
    int64_t rows, in_features, out_features;
    int32_t dtype, act;
    const void *x;        int64_t ldx;
    const void *weight;   int64_t ldw;
    const float *bias;
    const void *residual; int64_t ldr;
    void *y;              int64_t ldy;
    void *z;              int64_t ldz;
} ssd_linear_fwd;

/* Linear layer, backward:  dz = dy * act'(z),  dx = dz W,  dweight = dz^T x,  dbias = column sums of dz.
 * (The gradient of the residual is dy itself.)  dy, z [rows, out], x, dx [rows, in], weight [out, in] of
 * type `dtype`; dweight [out, in], dbias [out] of type `grad_dtype`.  Any of dx, dweight, dbias may be NULL;
 * x is not read without dweight, weight not without dx, z not when act is SSD_ACT_NONE (all may be NULL then).
 * With rows == 0 dweight and dbias are set to zero. */
typedef struct {
    int64_t rows, in_features, out_features;
    int32_t dtype, act, grad_dtype, reserved;
    const void *dy;       int64_t lddy;
    const void *x;        int64_t ldx;
    const void *weight;   int64_t ldw;
    const void *z;        int64_t ldz;
    void *dx;             int64_t lddx;
    void *dweight;        int64_t lddw;
    void *dbias;
} ssd_linear_bwd;

/* Gated projections, forward:  gate = x w_gate^T + b_gate,  up = x w_up^T + b_up,  h = act(gate) * up.
 * x [rows, in], w_gate, w_up [out, in], gate, up, h [rows, out] of type `dtype`; biases [out] float32.
 * b_gate, b_up, gate and up may be NULL (gate and up are what the backward pass needs). */
typedef struct {
    int64_t rows, in_features, out_features;
    int32_t dtype, act;
    const void *x;        int64_t ldx;
    const void *w_gate;   int64_t ldwg;
    const void *w_up;     int64_t ldwu;
    const float *b_gate;
    const float *b_up;
    void *h;              int64_t ldh;
    void *gate;           int64_t ldgate;
    void *up;             int64_t ldup;
} ssd_gated_fwd;

/* Gated projections, backward:  dgate = dh * up * act'(gate),  dup = dh * act(gate),
 * dx = dgate w_gate + dup w_up,  dw_gate = dgate^T x,  dw_up = dup^T x,  biases: column sums.
 * dw_gate and dw_up are given both or neither, and so are db_gate and db_up. */
typedef struct {
    int64_t rows, in_features, out_features;
    int32_t dtype, act, grad_dtype, reserved;
    const void *dh;       int64_t lddh;
    const void *x;        int64_t ldx;
    const void *w_gate;   int64_t ldwg;
    const void *w_up;     int64_t ldwu;
    const void *gate;     int64_t ldgate;
    const void *up;       int64_t ldup;
    void *dx;             int64_t lddx;
    void *dw_gate;        int64_t lddwg;
    void *dw_up;          int64_t lddwu;
    void *db_gate;
    void *db_up;
} ssd_gated_bwd;

/* Workspace that a call with these arguments needs, in bytes (0: none, NULL may be passed).  The pointers
 * are looked at for their alignment and for being NULL, not followed.  Errors as for the call itself, except that an
 * overlap is not looked for. */
ssd_status ssd_linear_forward_workspace(const ssd_linear_fwd *args, int64_t *bytes);
ssd_status ssd_linear_backward_workspace(const ssd_linear_bwd *args, int64_t *bytes);
ssd_status ssd_gated_forward_workspace(const ssd_gated_fwd *args, int64_t *bytes);
ssd_status ssd_gated_backward_workspace(const ssd_gated_bwd *args, int64_t *bytes);

/* The operators.  workspace: device memory of at least the bytes named above, 16-byte aligned.
 * Errors: SSD_ERR_ARG (NULL, sizes, pitches, unknown enum, overlap, workspace too small), SSD_ERR_ALIGN,
 * SSD_ERR_CUDA. */
ssd_status ssd_linear_forward(const ssd_linear_fwd *args, void *workspace, int64_t workspace_bytes, void *cuda_stream);
ssd_status ssd_linear_backward(const ssd_linear_bwd *args, void *workspace, int64_t workspace_bytes, void *cuda_stream);
ssd_status ssd_gated_forward(const ssd_gated_fwd *args, void *workspace, int64_t workspace_bytes, void *cuda_stream);
ssd_status ssd_gated_backward(const ssd_gated_bwd *args, void *workspace, int64_t workspace_bytes, void *cuda_stream);

/* Gradient norms over groups of tensors, and clipping.  For every group G of the list
 *     norm_G = sqrt(sum over the group's tensors of g^2)        (summed in double precision)
 *     c_G    = min(1, max_norm / (norm_G + 1e-6))
 *     out    = c_G * g                                          (one float32 product, rounded to dst_dtype)
 * A group is what is clipped together: one worker's whole gradient (K arenas, group i = worker i), every
 * tensor by itself, or all of them.
 *
 * ssd_grad_list: the tensors, made once for buffers that are used again and again.  numel: T element counts
 * (>= 0); group: T group numbers in 0..num_groups-1, in ascending order (NULL = all in group 0); a group without
 * tensors has norm 0.  src and dst: T device pointers of types src_dtype and dst_dtype; dst[t] == src[t]
 * clips in place (the types being equal); other overlaps are not allowed (SSD_ERR_ARG).  The arrays are copied.
 * `device_table`: caller-owned device memory of ssd_grad_list_bytes() bytes, 16-byte aligned, that the
 * kernels use for as long as the list lives; ssd_grad_list_create fills it by a copy on `cuda_stream` out of
 * the list's own (pageable) memory and waits for that copy, so that calls may follow on any stream.  (While the
 * stream is captured it does not wait: the copy is then part of the graph, and so are all calls on the list.)
 * Calls on one list must not overlap on the GPU: they share the table's space for partial sums.  The list and its
 * table outlive the calls on it, and the graphs that hold such calls. */
typedef struct ssd_grad_list ssd_grad_list;
ssd_status ssd_grad_list_bytes(int32_t num_tensors, const int64_t *numel, int32_t num_groups, int64_t *bytes);
ssd_status ssd_grad_list_create(ssd_grad_list **out, int32_t num_tensors, const int64_t *numel, const int32_t *group,
                                int32_t num_groups, const void *const *src, int32_t src_dtype, void *const *dst,
                                int32_t dst_dtype, void *device_table, int64_t table_bytes, void *cuda_stream);
void ssd_grad_list_destroy(ssd_grad_list *list);

/* What becomes of a group whose norm is infinite or NaN: its gradient is passed on as it is, or set to zero
 * so that the update sees nothing of it.  The norm reports it either way. */
typedef enum { SSD_NONFINITE_KEEP = 0, SSD_NONFINITE_ZERO = 1 } ssd_nonfinite;

/* norms: device array of num_groups floats, apart from gradients, destinations and table (SSD_ERR_ARG).  max_norm >= 0, or +infinity for no limit (dst is then a copy of src, or
 * left alone in place).  A group that needs no scaling is not written when in place. */
ssd_status ssd_clip_grad_norm(ssd_grad_list *list, float max_norm, int32_t nonfinite, float *norms, void *cuda_stream);

/* Norms alone: dst is not written. */
ssd_status ssd_grad_norm(ssd_grad_list *list, float *norms, void *cuda_stream);

/* 1 if a bounded wait inside a layer kernel ever ran out on the current device in this process (its results are then
 * incomplete); sticky; the call synchronises the device. */
ssd_status ssd_layer_error(int32_t *flag);

/* Text of the last CUDA error that a call of this header returned as SSD_ERR_CUDA on this host thread. */
const char *ssd_layer_cuda_error(void);

/* Kernels that the calls of this header have launched in this process. */
int64_t ssd_layer_launches(void);

#ifdef __cplusplus
}
#endif
#endif /* SSD_LAYERS_H */
