/*
 * merit_tokens.h -- operators along a sequence of tokens: a short causal convolution, a selective
 * state space scan, a group norm with an activation.  Forward and backward passes for whole
 * sequences, and the forms that continue a sequence by one token.
 *
 * All tensors are channels last: a token's channels lie side by side.  The convolution is a ranged
 * inner product, k = (b, t, d | a) with a moving along t at offset -(K-1); the scan is a recurrence
 * over its result; the norm closes the block (every token with statistics of its own), or normalises
 * an image that lies channels last (H * W positions share the statistics; the image layers of merit.h
 * leave planes, whose channels do not lie side by side).
 *
 * Conventions
 *   - An operand is a merit_view: a DEVICE pointer owned by the caller, the element strides of its
 *     two leading dimensions, its type.  Everything behind those two dimensions is dense.  Tensors
 *     of one or two dimensions without a leading batch are dense, their strides are not looked at.
 *     A leading stride may be anything for an input (a slice of a wider projection, 0 for a
 *     broadcast one).  data == NULL: absent, where the operand is optional.
 *   - Pointers are aligned to their element; on rows that start on 16-byte boundaries the norms
 *     move 16 bytes a lane and the convolutions four elements, else fewer.
 *   - "T" below is the plan's type: MERIT_F16, MERIT_BF16 or MERIT_F32.  "P": T or MERIT_F32.
 *     Arithmetic, sums, statistics and states are fp32 whatever T is; a result of type T is rounded
 *     once, to nearest even.
 *   - Outputs do not overlap inputs, but where a line below says so.
 *   - Work is enqueued on `hip_stream` and the call returns.  The library neither allocates nor
 *     synchronises; a pass that needs scratch memory takes it from the caller
 *     (merit_token_plan_workspace; 16-byte aligned; free for other use when the call's work is done).
 *   - A plan is immutable host memory, may be shared between threads and streams.
 *   - Results do not depend on the order in which workgroups run: the same call gives the same bits.
 *   - Sizes that a launch cannot hold are MERIT_ERR_UNSUPPORTED when the plan is made: fewer than 2^32
 *     threads a launch, which is 2^24 workgroups for most passes, and B L groups N < 2^31 for a scan.
 *   - Every function returns a merit_status; on an error nothing was launched (MERIT_ERR_HIP apart:
 *     of a call of several launches the first may have been).
 */
#ifndef MERIT_TOKENS_H
#define MERIT_TOKENS_H

#include "merit.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    void   *data;
    int64_t stride[2];
    int32_t dtype;           /* merit_dtype */
    int32_t reserved;        /* 0 */
} merit_view;

typedef enum { MERIT_ACT_NONE = 0, MERIT_ACT_RELU = 1, MERIT_ACT_SILU = 2 } merit_act;
typedef enum { MERIT_PASS_FORWARD = 0, MERIT_PASS_BACKWARD = 1, MERIT_PASS_STEP = 2 } merit_pass;

typedef struct merit_token_plan merit_token_plan;   /* opaque, host memory only */

#define MERIT_CONV_MAX_TAPS   8
#define MERIT_SCAN_MAX_STATES 64
#define MERIT_SCAN_TILE       16     /* tokens between two kept states of a forward pass */

/* Group norm of x[N, S, C]: the S positions x C / groups channels of a group share mean and variance.
 * S = 1: every token by itself; S = H * W: an image, channels last.  eps >= 0. */
merit_status merit_plan_group_norm(merit_dtype type, int64_t N, int64_t S, int64_t C, int64_t groups, double eps,
                                   merit_act act, merit_token_plan **out);
/* Causal convolution of x[B, L, D] with K <= MERIT_CONV_MAX_TAPS taps per channel. */
merit_status merit_plan_causal_conv(merit_dtype type, int64_t B, int64_t L, int64_t D, int64_t K, merit_act act,
                                    merit_token_plan **out);
/* Selective scan of x[B, L, D] with N <= MERIT_SCAN_MAX_STATES states per channel; the D / groups channels of
 * a group share the tokens' B and C.  softplus != 0: the step is log(1 + exp(dt + dt_bias)), else dt + dt_bias. */
merit_status merit_plan_scan(merit_dtype type, int64_t B, int64_t L, int64_t D, int64_t N, int64_t groups, int softplus,
                             merit_token_plan **out);
merit_status merit_token_plan_destroy(merit_token_plan *plan);
/* Scratch memory that a pass needs, in bytes (0: none). */
merit_status merit_token_plan_workspace(const merit_token_plan *plan, merit_pass pass, int64_t *bytes);
/* The kernels a pass runs ("a+b": two launches), for rows on 16-byte boundaries and with every gradient wanted but that
 * of `init`, which is a launch more (merit_cconv_dinit). */
merit_status merit_token_plan_kernel(const merit_token_plan *plan, merit_pass pass, const char **name);

/* y = act((x - mean) rstd weight + bias), rstd = 1 / sqrt(var + eps), var with the divisor S C / groups. */
typedef struct {
    merit_view x;            /* T [N, S, C]                                   */
    merit_view weight;       /* P [C], optional (1)                           */
    merit_view bias;         /* P [C], optional (0)                           */
    merit_view y;            /* T [N, S, C]; may be x                         */
    merit_view mean;         /* F32 [N, groups], optional: kept for backward  */
    merit_view rstd;         /* F32 [N, groups], optional                     */
} merit_group_norm_args;
merit_status merit_group_norm(const merit_token_plan *plan, const merit_group_norm_args *args, void *workspace,
                              int64_t workspace_bytes, void *hip_stream);

typedef struct {
    merit_view dy;           /* T [N, S, C]                                   */
    merit_view x;            /* T [N, S, C]                                   */
    merit_view mean;         /* F32 [N, groups], as the forward pass left it  */
    merit_view rstd;         /* F32 [N, groups]                               */
    merit_view weight;       /* P [C], optional                               */
    merit_view bias;         /* P [C], optional                               */
    merit_view dx;           /* T [N, S, C]; may be dy                        */
    merit_view dweight;      /* F32 [C], optional                             */
    merit_view dbias;        /* F32 [C], optional                             */
} merit_group_norm_backward_args;
merit_status merit_group_norm_backward(const merit_token_plan *plan, const merit_group_norm_backward_args *args,
                                       void *workspace, int64_t workspace_bytes, void *hip_stream);

/* y[b,t,d] = act(bias[d] + sum_a w[d,a] x[b, t-(K-1)+a, d]); the K-1 tokens before the first are `init`'s, or 0.
 * lens[b]: tokens of sequence b (cut to [0, L]); behind them x is not read and y is 0.
 * final: the last K-1 tokens of (init, x), the `init` of what follows. */
typedef struct {
    merit_view x;            /* T [B, L, D]                                   */
    merit_view weight;       /* P [D, K]                                      */
    merit_view bias;         /* P [D], optional (0)                           */
    merit_view init;         /* T [B, K-1, D], optional (0)                   */
    merit_view lens;         /* int32 [B], optional (L); its dtype is not looked at */
    merit_view y;            /* T [B, L, D]                                   */
    merit_view final;        /* T [B, K-1, D], optional; may be init          */
} merit_causal_conv_args;
merit_status merit_causal_conv(const merit_token_plan *plan, const merit_causal_conv_args *args, void *workspace,
                               int64_t workspace_bytes, void *hip_stream);

typedef struct {
    merit_view dy;           /* T [B, L, D]; not read behind lens             */
    merit_view x;            /* T [B, L, D]                                   */
    merit_view weight;       /* P [D, K]                                      */
    merit_view bias;         /* P [D], optional                               */
    merit_view init;         /* T [B, K-1, D], optional                       */
    merit_view lens;         /* int32 [B], optional                           */
    merit_view dfinal;       /* T [B, K-1, D], optional: gradient of `final`  */
    merit_view dx;           /* T [B, L, D]; 0 behind lens                    */
    merit_view dweight;      /* F32 [D, K], optional                          */
    merit_view dbias;        /* F32 [D], optional                             */
    merit_view dinit;        /* T [B, K-1, D], optional                       */
} merit_causal_conv_backward_args;
merit_status merit_causal_conv_backward(const merit_token_plan *plan, const merit_causal_conv_backward_args *args,
                                        void *workspace, int64_t workspace_bytes, void *hip_stream);

/* One more token of every sequence (the plan's L is not looked at). */
typedef struct {
    merit_view kept;         /* T [B, K-1, D]: the tokens before this one     */
    merit_view x;            /* T [B, D], stride[0] between sequences         */
    merit_view weight;       /* P [D, K]                                      */
    merit_view bias;         /* P [D], optional                               */
    merit_view y;            /* T [B, D], stride[0]                           */
    merit_view kept_out;     /* T [B, K-1, D]; may be kept                    */
} merit_causal_conv_step_args;
merit_status merit_causal_conv_step(const merit_token_plan *plan, const merit_causal_conv_step_args *args, void *workspace,
                                    int64_t workspace_bytes, void *hip_stream);

/* s = step(dt + dt_bias);  h_t[n] = exp(s A[n]) h_{t-1}[n] + s x B_t[n];  y = (sum_n C_t[n] h_t[n] + skip x) silu(z).
 * The states start from h0, or 0.  lens[b]: tokens of sequence b (cut to [0, L]); behind them nothing is read, y is 0
 * and the state stays.  h_last: the state behind the last token.  states: the states before every
 * MERIT_SCAN_TILE-th token, which the backward pass starts from. */
typedef struct {
    merit_view x;            /* T [B, L, D]                                   */
    merit_view dt;           /* T [B, L, D]                                   */
    merit_view A;            /* F32 [D, N]                                    */
    merit_view B;            /* T [B, L, groups, N]                           */
    merit_view C;            /* T [B, L, groups, N]                           */
    merit_view skip;         /* F32 [D], optional (0)                         */
    merit_view z;            /* T [B, L, D], optional (no gate)               */
    merit_view dt_bias;      /* F32 [D], optional (0)                         */
    merit_view h0;           /* F32 [B, D, N] dense, optional (0)             */
    merit_view lens;         /* int32 [B], optional                           */
    merit_view y;            /* T [B, L, D]                                   */
    merit_view h_last;       /* F32 [B, D, N] dense, optional                 */
    merit_view states;       /* F32 [B, ceil(L / MERIT_SCAN_TILE), D, N] dense, optional */
} merit_scan_args;
merit_status merit_scan(const merit_token_plan *plan, const merit_scan_args *args, void *workspace,
                        int64_t workspace_bytes, void *hip_stream);

typedef struct {
    merit_view dy;           /* T [B, L, D]; not read behind lens             */
    merit_view x;            /* T [B, L, D]                                   */
    merit_view dt;           /* T [B, L, D]                                   */
    merit_view A;            /* F32 [D, N]                                    */
    merit_view B;            /* T [B, L, groups, N]                           */
    merit_view C;            /* T [B, L, groups, N]                           */
    merit_view states;       /* F32, as the forward pass left them            */
    merit_view skip;         /* F32 [D], optional                             */
    merit_view z;            /* T [B, L, D], optional                         */
    merit_view dt_bias;      /* F32 [D], optional                             */
    merit_view lens;         /* int32 [B], optional                           */
    merit_view dh_last;      /* F32 [B, D, N] dense, optional: gradient of h_last */
    merit_view dx;           /* T [B, L, D]; these four: 0 behind lens        */
    merit_view ddt;          /* T [B, L, D]                                   */
    merit_view dB;           /* T [B, L, groups, N]                           */
    merit_view dC;           /* T [B, L, groups, N]                           */
    merit_view dz;           /* T [B, L, D]; present where z is               */
    merit_view dA;           /* F32 [D, N]                                    */
    merit_view dskip;        /* F32 [D], optional                             */
    merit_view ddt_bias;     /* F32 [D], optional                             */
    merit_view dh0;          /* F32 [B, D, N] dense, optional                 */
} merit_scan_backward_args;
merit_status merit_scan_backward(const merit_token_plan *plan, const merit_scan_backward_args *args, void *workspace,
                                 int64_t workspace_bytes, void *hip_stream);

/* One more token of every sequence (the plan's L is not looked at).  Two-dimensional operands: stride[0]. */
typedef struct {
    merit_view h;            /* F32 [B, D, N] dense                           */
    merit_view x;            /* T [B, D]                                      */
    merit_view dt;           /* T [B, D]                                      */
    merit_view A;            /* F32 [D, N]                                    */
    merit_view B;            /* T [B, groups, N]                              */
    merit_view C;            /* T [B, groups, N]                              */
    merit_view skip;         /* F32 [D], optional                             */
    merit_view z;            /* T [B, D], optional                            */
    merit_view dt_bias;      /* F32 [D], optional                             */
    merit_view y;            /* T [B, D]                                      */
    merit_view h_out;        /* F32 [B, D, N] dense; may be h                 */
} merit_scan_step_args;
merit_status merit_scan_step(const merit_token_plan *plan, const merit_scan_step_args *args, void *workspace,
                             int64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MERIT_TOKENS_H */
