/*
 * lbi_block.h -- C-ABI of the operators of a state-space region block on
 * MI355X (gfx950), in the same library as lbi.h.
 *
 * The architecture section of LBI lists state-space models among the region
 * transformations Phi_k.  Between its projections such a block consists of
 * three operators over the tokens of a batch, given here with the forms that
 * training, prompts and single decoded tokens need:
 *
 *   norm   s = x + residual,  out = s / sqrt(mean(s^2) + eps) * weight,
 *          in the token type or in 8 bits with scales; its gradient.
 *   conv   out_t = f(bias + sum_w weight_w x_{t-W+1+w}) along the tokens of a
 *          sequence, channel by channel, f = silu or the identity; its
 *          gradient; its form for one token a sequence.
 *   scan   h_t = exp(D_t A) h_{t-1} + D_t u_t B_t  (channel d, state n),
 *          y_t = (sum_n C_t h_t + skip u_t) silu(z_t),
 *          D_t = softplus(delta_t + delta_bias); its gradient; its form for
 *          one token a sequence.
 *
 * Conventions, in addition to those of lbi.h (asynchronous on `stream`, no
 * allocation, argument errors before anything is enqueued):
 *   - Token tensors hold one row a token, `dt` values, at a row stride `ld`
 *     (in elements, at least the row's length): halves and slices of a
 *     projection's output are passed as they are.  Pointers need the
 *     alignment of their elements only; rows may start anywhere.
 *   - A batch of sequences is packed: the T rows of all of them back to back.
 *     `offsets` is a DEVICE array of B + 1 int64 values, offsets[0] = 0 and
 *     offsets[B] = T, sequence i being rows offsets[i] .. offsets[i+1] - 1; a
 *     sequence may be empty.  NULL: B sequences of T / B rows each.  The
 *     contents are read on the GPU and cannot be refused: what does not
 *     ascend from 0 to T gives wrong results, within the given tensors.
 *   - Parameters that belong to a channel, states of the scan and the
 *     gradients of both are float32.  Sums, states and norms are held in
 *     float32 for every dt; each output is rounded once.
 *   - `slots`: a DEVICE array of one int32 a sequence, or NULL.  Row slots[i]
 *     of state_in and state_out (n_slots rows) belongs to sequence i; NULL:
 *     row i.  A slot outside 0 .. n_slots - 1 means no state: zeros are read
 *     and nothing is written.  No two sequences may share a slot.
 *   - state_out may be the same pointer as state_in.  No other output may
 *     overlap an input, the workspace or another output (LBI_ERR_ALIAS).
 *   - Results do not depend on timing: the same call gives the same bits.
 *   - Sizes of zero (T = 0, B = 0) are valid; with T = 0 only states,
 *     gradients of states and (zero) gradients of parameters are written.
 */
#ifndef LBI_BLOCK_H
#define LBI_BLOCK_H

#include "lbi.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LBI_NORM_MAX_D 16384 /* longest row of the norm                        */
#define LBI_SSM_MAX_D 65536  /* most channels of the convolution and the scan  */
#define LBI_SSM_MAX_N 64     /* most states of a channel                       */
#define LBI_SSM_MAX_LD (1 << 23) /* longest row stride of their token tensors  */
#define LBI_CONV_MAX_W 4     /* most taps of the convolution                   */

/* Formats of an 8-bit output. */
typedef enum {
    LBI_Q8_E4M3 = 0, /* 4 exponent and 3 mantissa bits, largest value 448, no
                      * infinities (torch.float8_e4m3fn)                      */
    LBI_Q8_INT8 = 1  /* signed integers -127 .. 127                           */
} lbi_q8_format;

/*
 * Root-mean-square norm with the residual's addition.
 *
 *   x             [T][D] dt.
 *   residual      [T][D] residual_dt, or NULL (no addition).
 *   weight        [D] float32.
 *   out           OUTPUT [T][D] dt: s * rsqrt(mean(s^2) + eps) * weight, with
 *                 s = x + residual in float32 (not yet rounded).
 *   residual_out  OUTPUT [T][D] residual_dt: s, or NULL (not written; then
 *                 required to be NULL without a residual).
 *   T >= 0, 1 <= D <= LBI_NORM_MAX_D, eps >= 0 (else LBI_ERR_SHAPE).
 * residual_out may be the same pointer as residual (with the same stride).
 * A row of zeros gives zeros (eps > 0); a NaN or an infinity gives NaN in its
 * row.  The sum of the squares is float32: where it passes that range (values
 * of 10^19 / sqrt(D) and more) finite values give zeros.
 */
lbi_status lbi_rms_norm(const void *x, int64_t ld_x, const void *residual, int64_t ld_residual,
                        const float *weight, void *out, int64_t ld_out, void *residual_out,
                        int64_t ld_residual_out, int64_t T, int32_t D, float eps, lbi_dtype dt,
                        lbi_dtype residual_dt, lbi_stream_t stream);

/*
 * The same norm with its output in 8 bits: out = q * scale.
 *
 *   q       OUTPUT [T][D] bytes, at row stride ld_q: out / scale rounded to
 *           the nearest value of `format` (ties to even).
 *   scales  OUTPUT [T][ceil(D / group)] float32, dense: the largest |out| of
 *           the group's features times the float32 value of 1 / 448 (E4M3) or
 *           1 / 127 (INT8).  1 where that is below the smallest normal float32
 *           (q is then 0), NaN where an out of the group is NaN or infinite.
 *   group   features that share a scale: 32, 64 or 128, or 0 for the whole row
 *           (else LBI_ERR_SHAPE).
 *   format  an lbi_q8_format (else LBI_ERR_DTYPE).
 *
 * A quotient in the middle between two values of the format goes by the last
 * bits of what it was computed from.  So each operation here is rounded to
 * float32 by itself, (s * rsqrt(sum * (1 / D) + eps)) * weight, and the sum of
 * the squares has a stated order.  D < 128: sum l of L = min(64, the largest
 * power of two up to D) is that of elements l and l + L.  D >= 128: the row's
 * aligned vectors of four, which begin where t D + d is a multiple of four, go
 * to 64 lanes (32 for D < 256, 512 for D > 8128) in turn; a lane's four sums
 * (one an element of its vectors) grow along the row and are added in order;
 * what lies ahead of the first vector or after the last joins the first sum of
 * lanes (t D mod 4) .. 3 and 0 .. 2.  The lanes' sums are added pairwise,
 * neighbours first, up to 64 of them, and the eight that this leaves of 512 by
 * halves, the first with the fifth.  (For D no multiple of four a row's last
 * bits go by its place t.)
 */
lbi_status lbi_rms_norm_q8(const void *x, int64_t ld_x, const void *residual,
                           int64_t ld_residual, const float *weight, void *q, int64_t ld_q,
                           float *scales, void *residual_out, int64_t ld_residual_out, int64_t T,
                           int32_t D, float eps, int32_t group, lbi_q8_format format,
                           lbi_dtype dt, lbi_dtype residual_dt, lbi_stream_t stream);

/*
 * Gradient of the norm.
 *
 *   dout       [T][D] dt: gradient of out.
 *   s          [T][D] residual_dt: what was normalised (residual_out of the
 *              forward call, or x where there was no residual).
 *   dresidual  [T][D] residual_dt, or NULL (= 0): gradient that reaches s past
 *              the norm (of residual_out).
 *   ds         OUTPUT [T][D] residual_dt: gradient of s, that is of x and of
 *              residual alike:  r (g - n mean(g n)) + dresidual  with
 *              r = rsqrt(mean(s^2) + eps), n = s r, g = dout weight.  May be
 *              the same pointer as dresidual (with the same stride).
 *   dweight    OUTPUT [D] float32: the sum over rows of dout n; or NULL.
 *   workspace  lbi_rms_norm_backward_workspace_bytes(T, D) bytes, 256-byte
 *              aligned (partial sums of dweight; unused when dweight is NULL).
 */
size_t lbi_rms_norm_backward_workspace_bytes(int64_t T, int32_t D);
lbi_status lbi_rms_norm_backward(const void *dout, int64_t ld_dout, const void *s, int64_t ld_s,
                                 const float *weight, const void *dresidual,
                                 int64_t ld_dresidual, void *ds, int64_t ld_ds, float *dweight,
                                 int64_t T, int32_t D, float eps, lbi_dtype dt,
                                 lbi_dtype residual_dt, void *workspace, size_t workspace_bytes,
                                 lbi_stream_t stream);

/*
 * Short causal convolution along the tokens, channel by channel.
 *
 *   x          [T][D] dt, packed sequences.
 *   weight     [D][W] float32; weight[d][W-1] multiplies the token itself.
 *   bias       [D] float32, or NULL (= 0).
 *   out        OUTPUT [T][D] dt.
 *   state_in   [B or n_slots][W-1][D] dt: the W - 1 tokens before each
 *              sequence, oldest first, or NULL (zeros).
 *   state_out  OUTPUT, as state_in: the last W - 1 tokens of state_in and the
 *              sequence together, exact copies; or NULL (not written).
 *   silu       0: out is the plain sum; otherwise its silu.
 *   2 <= W <= LBI_CONV_MAX_W, 1 <= D <= LBI_SSM_MAX_D, T a multiple of B without offsets.
 */
lbi_status lbi_ssm_conv(const void *x, int64_t ld_x, const float *weight, const float *bias,
                        void *out, int64_t ld_out, const void *state_in, void *state_out,
                        const int32_t *slots, int32_t n_slots, const int64_t *offsets, int64_t T,
                        int64_t B, int32_t D, int32_t W, int32_t silu, lbi_dtype dt,
                        lbi_stream_t stream);

/*
 * Gradient of lbi_ssm_conv (states by sequence, without slots).
 *
 *   dout        [T][D] dt.
 *   dstate_out  [B][W-1][D] dt: gradient of state_out, or NULL (= 0).
 *   dx          OUTPUT [T][D] dt.
 *   dweight     OUTPUT [D][W] float32.
 *   dbias       OUTPUT [D] float32, or NULL.
 *   dstate_in   OUTPUT [B][W-1][D] dt, or NULL.
 *   workspace   lbi_ssm_conv_backward_workspace_bytes(T, D, W) bytes, 256-byte
 *               aligned.
 */
size_t lbi_ssm_conv_backward_workspace_bytes(int64_t T, int32_t D, int32_t W);
lbi_status lbi_ssm_conv_backward(const void *x, int64_t ld_x, const float *weight,
                                 const float *bias, const void *dout, int64_t ld_dout,
                                 const void *state_in, const void *dstate_out, void *dx,
                                 int64_t ld_dx, float *dweight, float *dbias, void *dstate_in,
                                 const int64_t *offsets, int64_t T, int64_t B, int32_t D,
                                 int32_t W, int32_t silu, lbi_dtype dt, void *workspace,
                                 size_t workspace_bytes, lbi_stream_t stream);

/*
 * One token for each of n sequences: x and out [n][D]; state_in and state_out
 * (both required, may be the same) as for lbi_ssm_conv.  A sequence whose slot
 * is out of range is computed from zeros, and its state is not written.
 */
lbi_status lbi_ssm_conv_step(const void *x, int64_t ld_x, const float *weight, const float *bias,
                             void *out, int64_t ld_out, const void *state_in, void *state_out,
                             const int32_t *slots, int32_t n_slots, int64_t n, int32_t D,
                             int32_t W, int32_t silu, lbi_dtype dt, lbi_stream_t stream);

/* What the forms of the scan read (a HOST struct of DEVICE pointers). */
typedef struct {
    const void *u;           /* [T][D] dt                                     */
    int64_t ld_u;
    const void *delta;       /* [T][D] dt                                     */
    int64_t ld_delta;
    const void *z;           /* [T][D] dt, or NULL (no gate)                  */
    int64_t ld_z;
    const void *B;           /* [T][G][N] dt, a token's G N values dense      */
    int64_t ld_B;
    const void *C;           /* [T][G][N] dt                                  */
    int64_t ld_C;
    const float *A;          /* [D][N]; exp(D_t A) decays where A < 0.  A > 0:
                              * states and outputs are as token by token; the
                              * gradient of a state before tokens that together
                              * grow it by 2^127 may be infinite or NaN       */
    const float *skip;       /* [D], or NULL (= 0)                            */
    const float *delta_bias; /* [D], or NULL (= 0)                            */
    const float *state_in;   /* [sequences or n_slots][D][N], or NULL (zeros) */
    const int64_t *offsets;  /* [sequences + 1] DEVICE, or NULL               */
    int64_t T;               /* tokens of all sequences                       */
    int64_t sequences;       /* fewer than 2^32                               */
    int32_t D;               /* channels                                      */
    int32_t N;               /* states of a channel, 1 .. LBI_SSM_MAX_N       */
    int32_t G;               /* groups: channels g D/G .. share B and C; G
                              * divides D                                     */
    int32_t softplus;        /* 0: D_t = delta_t + delta_bias as it is        */
    lbi_dtype dt;
} lbi_ssm_inputs;

/*
 * The selective scan over packed sequences.
 *
 *   y          OUTPUT [T][D] dt, at row stride ld_y.
 *   state_out  OUTPUT, as state_in: the states after each sequence's last
 *              token; or NULL.
 *   workspace  lbi_ssm_scan_workspace_bytes(...) bytes, 256-byte aligned (NULL
 *              where that is 0).  ragged: offsets given.
 */
size_t lbi_ssm_scan_workspace_bytes(int64_t T, int64_t sequences, int32_t D, int32_t N,
                                    int32_t G, int32_t ragged);
lbi_status lbi_ssm_scan(const lbi_ssm_inputs *in, void *y, int64_t ld_y, float *state_out,
                        const int32_t *slots, int32_t n_slots, void *workspace,
                        size_t workspace_bytes, lbi_stream_t stream);

/* What lbi_ssm_scan_backward writes (a HOST struct of DEVICE pointers). */
typedef struct {
    void *du;            /* [T][D] dt                                         */
    int64_t ld_du;
    void *ddelta;        /* [T][D] dt                                         */
    int64_t ld_ddelta;
    void *dz;            /* [T][D] dt; required with z, else NULL             */
    int64_t ld_dz;
    void *dB;            /* [T][G][N] dt                                      */
    int64_t ld_dB;
    void *dC;            /* [T][G][N] dt                                      */
    int64_t ld_dC;
    float *dA;           /* [D][N]                                            */
    float *dskip;        /* [D], or NULL                                      */
    float *ddelta_bias;  /* [D], or NULL                                      */
    float *dstate_in;    /* [sequences][D][N], or NULL                        */
} lbi_ssm_gradients;

/*
 * Gradient of lbi_ssm_scan (states by sequence, without slots), from the
 * forward's inputs alone: the states are computed again.
 *
 *   dy          [T][D] dt.
 *   dstate_out  [sequences][D][N] float32: gradient of state_out, or NULL.
 */
size_t lbi_ssm_scan_backward_workspace_bytes(int64_t T, int64_t sequences, int32_t D, int32_t N,
                                             int32_t G, int32_t ragged);
lbi_status lbi_ssm_scan_backward(const lbi_ssm_inputs *in, const void *dy, int64_t ld_dy,
                                 const float *dstate_out, const lbi_ssm_gradients *grads,
                                 void *workspace, size_t workspace_bytes, lbi_stream_t stream);

/*
 * One token for each of in->sequences sequences (in->T must equal it and
 * in->offsets be NULL, else LBI_ERR_SHAPE); in->state_in and state_out are
 * both required and may be the same.  A sequence whose slot is out of range is
 * computed from zeros, and its state is not written.
 */
lbi_status lbi_ssm_scan_step(const lbi_ssm_inputs *in, void *y, int64_t ld_y, float *state_out,
                             const int32_t *slots, int32_t n_slots, lbi_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* LBI_BLOCK_H */
