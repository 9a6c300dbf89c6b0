/*
 * rps_ops.h: C ABI of the training operators that stand next to the RPS step (rps.h), on one NVIDIA B200 (sm_100a).
 *
 * The RPS step averages the replicas of n simulated workers; these operators make the gradient that a worker's own step
 * needs when the model is a network with a large output vocabulary (the paper trains a language model among others,
 * Section 5).  All n workers go through one call: every array has a leading worker axis, and parameters are read out
 * of (and their gradients may be written into) rows of an [n][pitch] array such as rps_bind() takes.
 *
 * General rules
 *   - Every function returns RPS_OK or a negative rps_status; nothing throws or aborts.  rps_ops_last_error() gives a
 *     readable reason for the last failure on the calling thread.
 *   - There is no handle and no state between calls.  Calls on different streams or host threads are independent as
 *     long as they are given different workspaces and outputs.
 *   - All array arguments are device pointers of the current device, owned by the caller.  The library allocates no
 *     device memory: a call that needs scratch says how much (..._workspace) and is lent it, 256-byte aligned; its
 *     contents mean nothing before or after the call.
 *   - Work is enqueued on cuda_stream (a cudaStream_t, NULL = the default stream) and nothing waits for it: errors of
 *     execution surface at the caller's next synchronising call.  Calls may be captured into a CUDA graph after one call
 *     outside it (the first call on a device asks the driver for attributes).
 *   - dtype is an rps_dtype: RPS_F32 or RPS_BF16, one type for all arrays of a call that are not said to be something
 *     else.  Sums, statistics and accumulators are fp32; a bf16 result is rounded once, at the store, unless a comment
 *     says otherwise.  The tensor cores cut their sums off instead of rounding them, so those go through in runs that are added in
 *     fp32, rounded: of 128 terms with RPS_F32 (whose products leave out less than 2^-24 of themselves), of 1024 for the loss and
 *     32768 for the gradients with RPS_BF16.  Infinities and NaN go through matrix products as they do through fp32 arithmetic,
 *     but for two cases of RPS_F32: an infinity times an infinity is NaN, and where dloss is infinite the gradients are either
 *     infinite or NaN.  Results do not depend on the order in which blocks run: no call uses floating-point atomics.
 *   - Strides are in elements, and the innermost axis is always contiguous.  Sizes may be zero where a comment says so.
 */
#ifndef RPS_OPS_H
#define RPS_OPS_H

#include "rps.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    RPS_PACK_GROUP = 128,       /* consecutive columns of a row that share one scale in 8-bit activations */
    RPS_MAX_NORM_COLS = 16384   /* widest row of rps_norm_forward / rps_norm_backward                     */
};

/* ------------------------------------------------------------------------------------------------------------------
 * Softmax cross entropy of a linear layer over a large vocabulary, without keeping the logits.
 *
 *   l[t][v] = sum_c hidden[t][c] * weight[v][c]
 *   lse[t]  = log sum_v exp(l[t][v])
 *   loss[t] = lse[t] - l[t][target[t]]
 *   dl[t][v] = g[t] * (exp(l[t][v] - lse[t]) - [v == target[t]])
 *   dhidden = dl * weight,   dweight = dl^T * hidden
 *
 * for each worker by itself.  The vocabulary goes through in pieces; the logits of a tile exist on the SM alone, and
 * the backward pass makes them again, holding dl (rounded to bf16, or as three bf16 parts that add up to 24 bits for
 * RPS_F32) for one piece at a time in the workspace.
 *
 * Tokens whose target is ignore_index take no part: their rows of hidden are not read (they may hold anything, NaN and
 * infinities included), their loss and lse are 0 and their row of dhidden is 0; the work shrinks with their number.
 * Any other target outside 0..vocab-1 is a mistake of the caller that the host cannot see: it gives that token's
 * loss, and every gradient it takes part in, the value NaN.
 * ------------------------------------------------------------------------------------------------------------------ */
typedef enum rps_reduction {
    RPS_REDUCE_NONE = 0, /* loss and dloss are [n][tokens]                                              */
    RPS_REDUCE_SUM = 1,  /* loss and dloss are [n]: the sum over a worker's tokens                      */
    RPS_REDUCE_MEAN = 2  /* [n]: the sum divided by the number of tokens that are not ignored; 0 (and no
                            gradient) for a worker that has none                                        */
} rps_reduction;

typedef struct rps_lce_desc {
    int32_t dtype;         /* of hidden, weight, dhidden, dweight                                        */
    int32_t reduction;     /* rps_reduction                                                              */
    int32_t n;             /* workers, 1..RPS_MAX_WORKERS                                                */
    int64_t tokens;        /* tokens of a worker, 0 <= tokens < 2^24                                     */
    int64_t vocab;         /* rows of weight, 1 <= vocab < 2^30                                          */
    int64_t cols;          /* width of hidden and weight, 1 <= cols < 2^24                               */
    int64_t ignore_index;
    int64_t hidden_row, hidden_worker;   /* strides of hidden; hidden_row >= cols                        */
    int64_t weight_row, weight_worker;   /* strides of weight; weight_row >= cols                        */
    int64_t dweight_row, dweight_worker; /* strides of dweight (backward only); cols <= dweight_row < 2^31 */
} rps_lce_desc;

/* Bytes of workspace that rps_lce_forward (backward = 0) or rps_lce_backward (backward = 1) wants.  Of the weight only
 * the address counts: one that is not 16-byte aligned (or has such strides) is laid out anew, piece by piece.          */
int rps_lce_workspace(const rps_lce_desc* desc, const void* weight, int backward, size_t* bytes);

/* targets: int64 [n][tokens], dense.  loss: float, as reduction says.  lse: float [n][tokens], dense, for the backward
 * pass.  Both outputs are written whole.                                                                              */
int rps_lce_forward(const rps_lce_desc* desc, const void* hidden, const void* weight, const int64_t* targets, float* loss,
                    float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* dloss: float, shaped as loss.  lse: what the forward pass of the same inputs wrote.  dhidden: [n][tokens][cols], dense.
 * dweight: vocab rows of cols for each worker, at its strides; what lies between the rows is not touched.  Both are
 * written, not added to.                                                                                              */
int rps_lce_backward(const rps_lce_desc* desc, const void* hidden, const void* weight, const int64_t* targets,
                     const float* lse, const float* dloss, void* dhidden, void* dweight, void* workspace,
                     size_t workspace_bytes, void* cuda_stream);

/* ------------------------------------------------------------------------------------------------------------------
 * The step between two blocks of a network: norm after the block, gate, residual scale, residual sum, norm before the
 * next block.  With r(z) = 1 / sqrt(mean(z^2) + eps) of a row:
 *
 *   u = f * r(f) * post            f: the block's output
 *   h = x + scale * gate * u       x: the residual stream; h: the residual stream after the block
 *   y = h * r(h) * pre             y: the next block's input
 *
 * gate has `gates` rows for a worker's tokens, gates a divisor of tokens: consecutive runs of tokens / gates tokens share
 * a row (1: a gate for each channel; tokens: for each token and channel; otherwise one for each sequence).
 *
 *   t = dh + r(h) * (a - h * r(h)^2 * mean(a * h)),   a = dy * pre
 *   dx = t,   df = r(f) * (b - f * r(f)^2 * mean(b * f)),   b = scale * gate * t * post
 *   dgate = sum scale * u * t,  dpost = sum scale * gate * t * f * r(f),  dpre = sum dy * h * r(h)
 *
 * x, f, h, y and their gradients are dense [n][tokens][cols]; post and pre are [n][cols] with a stride between workers,
 * gate is [n][gates][cols] with a stride between workers.  The backward pass reads f and h either as they are stored (h of
 * RPS_BF16 rounded, that is, while r(h) and y are made of h before it is) or as 8-bit codes of that with scales (rps_pack), which the
 * forward pass writes along the way when it is given room for them; r(f) and r(h) are always those of the values before rounding and
 * packing.  tokens may be 0; n * tokens < 2^31.
 * ------------------------------------------------------------------------------------------------------------------ */
typedef struct rps_norm_desc {
    int32_t dtype;
    int32_t n;               /* workers, 1..RPS_MAX_WORKERS                           */
    int64_t tokens;          /* tokens of a worker, 0 <= n * tokens < 2^31            */
    int64_t cols;            /* 1..RPS_MAX_NORM_COLS                                  */
    int64_t gates;           /* rows of gate, a divisor of tokens (1 if tokens is 0)  */
    int64_t post_worker, pre_worker, gate_worker;    /* strides between workers       */
    double scale;            /* finite                                                */
    double eps;              /* >= 0                                                  */
    int32_t wait_limit_ms;   /* rows wider than a CTA holds (8 KB) are shared by CTAs that wait for one another's sums; every such
                                wait gives up after this many milliseconds (0 = 2000) */
    int32_t withhold_sums;   /* test aid for that: 1 = one CTA of each row sends no sums, so the others' waits run out, the rows'
                                results are not written and rps_ops_check reports it; 0 otherwise */
} rps_norm_desc;

/* r_f, r_h: float [n][tokens], written for the backward pass; both may be NULL together.  f_codes, f_scales, h_codes,
 * h_scales: room for 8-bit copies of f and of h (as stored) in the form of rps_pack with n * tokens rows; all four or
 * none (NULL).                                                                                                      */
int rps_norm_forward(const rps_norm_desc* desc, const void* x, const void* f, const void* gate, const void* post,
                     const void* pre, void* h, void* y, float* r_f, float* r_h, int8_t* f_codes, float* f_scales,
                     int8_t* h_codes, float* h_scales, void* cuda_stream);

/* Bytes of workspace that rps_norm_backward wants. */
int rps_norm_workspace(const rps_norm_desc* desc, size_t* bytes);

/* f, h: the tensors themselves with f_scales = h_scales = NULL, or the codes with their scales (both or neither packed).
 * dh may be NULL (no gradient reaches h but through y).  dgate, dpost and dpre are dense: [n][gates][cols], [n][cols],
 * [n][cols].                                                                                                        */
int rps_norm_backward(const rps_norm_desc* desc, const void* dh, const void* dy, const void* f, const float* f_scales,
                      const void* h, const float* h_scales, const float* r_f, const float* r_h, const void* gate,
                      const void* post, const void* pre, void* dx, void* df, void* dgate, void* dpost, void* dpre,
                      void* workspace, size_t workspace_bytes, void* cuda_stream);

/* ------------------------------------------------------------------------------------------------------------------
 * Activations kept in 8 bits.  Each run of RPS_PACK_GROUP consecutive columns of a row (the last one may be short) has
 *
 *   scale = max|x| * (1/127),   code = rint(x * (127 / max|x|)),   and stands for  code * scale
 *
 * with every operation rounded to fp32 (ties of rint to even).  A group whose max|x| is below 2^-100 has scale 0 and
 * codes 0; a group that holds an infinity or a NaN has scale NaN, so all of it reads back as NaN.
 * codes: int8 [rows][rps_pack_pitch(cols)], the columns past cols zero; scales: float [rows][ceil(cols / RPS_PACK_GROUP)].
 * codes and scales are 16-byte aligned.
 * ------------------------------------------------------------------------------------------------------------------ */
int64_t rps_pack_pitch(int64_t cols); /* cols rounded up to a multiple of 16 */

/* x: rows of cols elements, x_row elements apart (x_row >= cols).  rows may be 0; cols 1..2^24-1. */
int rps_pack(int dtype, int64_t rows, int64_t cols, const void* x, int64_t x_row, int8_t* codes, float* scales,
             void* cuda_stream);
int rps_unpack(int dtype, int64_t rows, int64_t cols, const int8_t* codes, const float* scales, void* x, int64_t x_row,
               void* cuda_stream);

/* Weight gradient of a linear layer out of its packed input, for each worker:  dweight[o][c] = sum_t dy[t][o] * x[t][c],
 * x the values that codes and scales (of n * tokens rows) stand for; with RPS_BF16 those are rounded to bf16 on the way
 * into the tensor cores, which is the precision of dy.                                                              */
typedef struct rps_wgrad_desc {
    int32_t dtype;           /* of dy and dweight                                     */
    int32_t n;               /* workers, 1..RPS_MAX_WORKERS                           */
    int64_t tokens;          /* 0 <= tokens < 2^24, n * tokens < 2^31                 */
    int64_t outs, cols;      /* 1..2^24-1                                             */
    int64_t dy_row, dy_worker, dweight_row, dweight_worker; /* strides; rows >= outs and >= cols, dweight_row < 2^31 */
    int32_t wait_limit_ms;   /* every wait of the product's kernel on data gives up after this many milliseconds (0 = 2000) */
    int32_t withhold_copies; /* test aid for that: 1 = the kernel issues no copies, so its waits run out, the result is not
                                written and rps_ops_check reports it; 0 otherwise                                           */
} rps_wgrad_desc;

/* Of dy only the address counts. */
int rps_wgrad_workspace(const rps_wgrad_desc* desc, const void* dy, size_t* bytes);
int rps_packed_wgrad(const rps_wgrad_desc* desc, const void* dy, const int8_t* codes, const float* scales, void* dweight,
                     void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Every wait inside a kernel is bounded (two seconds, unless a description says otherwise): those of the matrix products on data, and those of the
 * norms whose rows are shared by several CTAs on one another's sums.  One that gives up ends its kernel early; what the call had
 * not written by then is not written, and what it has written is not valid.  rps_ops_check synchronises the stream and returns
 * RPS_ECUDA if that happened on the current device since the last check. */
int rps_ops_check(void* cuda_stream);

/* Reason for the last failure of a function of this file on the calling thread ("" if none). */
const char* rps_ops_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* RPS_OPS_H */
