/*
 * lbi_linear.h -- C-ABI of the operators of a region block with linear
 * attention on MI355X (gfx950), in the same library as lbi.h and lbi_block.h.
 *
 * The architecture section of LBI leaves the region transformations Phi_k open
 * and has layer norms and two-layer maps at the interfaces.  Where lbi_block.h
 * has a state-space block between its projections, this header has a block
 * whose tokens mix by linear attention, its norm, and the projections:
 *
 *   layer norm        s = x + residual,
 *                     out = (s - mean(s)) / sqrt(var(s) + eps) * weight + bias;
 *                     its gradient.
 *   projection        out = act(x W^T + bias) + residual in one pass over the
 *                     product; its gradient.
 *   linear attention  S_t = a S_{t-1} + k_t v_t^T,  o_t = scale q_t^T S_t, with
 *                     a = exp(log_decay) for each head: causal attention without
 *                     a softmax whose weights fade with the distance; its
 *                     gradient; its form for one token a sequence.
 *
 * Conventions: those of lbi.h and lbi_block.h (token rows at a stride, packed
 * sequences with offsets on the device, states in slots, no allocation, argument
 * errors before anything is enqueued, results that do not depend on timing).
 */
#ifndef LBI_LINEAR_H
#define LBI_LINEAR_H

#include "lbi_block.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LBI_PROJECTION_MAX 65536    /* most features of a projection, in or out     */
#define LBI_ATTENTION_MAX_DIM 128   /* longest key and longest value of a head      */
#define LBI_ATTENTION_MAX_H 1024    /* most heads                                   */
#define LBI_ATTENTION_MAX_LD (1 << 23) /* longest row stride of the tensors it reads  */

/*
 * Layer norm with the residual's addition.
 *
 *   x, residual, residual_out  as for lbi_rms_norm: s = x + residual.
 *   weight        [D] float32, or NULL (= 1).
 *   bias          [D] float32, or NULL (= 0).
 *   out           OUTPUT [T][D] dt: (s - mean(s)) * rsqrt(var(s) + eps) * weight + bias, with
 *                 var(s) = mean((s - mean(s))^2) and s in float32 (not yet rounded).
 *   T >= 0, 1 <= D <= LBI_NORM_MAX_D, eps >= 0 (else LBI_ERR_SHAPE).
 * A row of equal values gives bias (eps > 0); a NaN or an infinity gives NaN in
 * its row, as does a difference from the mean that float32 does not hold.  The
 * sum of the squares is float32: where it passes that range (differences of
 * 10^19 / sqrt(D) and more) finite values give bias, and a gradient of dresidual.
 */
lbi_status lbi_layer_norm(const void *x, int64_t ld_x, const void *residual, int64_t ld_residual,
                          const float *weight, const float *bias, void *out, int64_t ld_out,
                          void *residual_out, int64_t ld_residual_out, int64_t T, int32_t D,
                          float eps, lbi_dtype dt, lbi_dtype residual_dt, lbi_stream_t stream);

/*
 * Gradient of the layer norm; dout, s, dresidual and ds as for
 * lbi_rms_norm_backward.
 *
 *   ds         OUTPUT: r (g - mean(g) - n mean(g n)) + dresidual  with
 *              r = rsqrt(var(s) + eps), n = (s - mean(s)) r, g = dout weight.
 *   dweight    OUTPUT [D] float32: the sum over rows of dout n; or NULL.
 *   dbias      OUTPUT [D] float32: the sum over rows of dout; or NULL.
 *   workspace  lbi_layer_norm_backward_workspace_bytes(T, D) bytes, 256-byte
 *              aligned (unused when dweight and dbias are NULL).
 */
size_t lbi_layer_norm_backward_workspace_bytes(int64_t T, int32_t D);
lbi_status lbi_layer_norm_backward(const void *dout, int64_t ld_dout, const void *s, int64_t ld_s,
                                   const float *weight, const void *dresidual,
                                   int64_t ld_dresidual, void *ds, int64_t ld_ds, float *dweight,
                                   float *dbias, int64_t T, int32_t D, float eps, lbi_dtype dt,
                                   lbi_dtype residual_dt, void *workspace, size_t workspace_bytes,
                                   lbi_stream_t stream);

/* What a projection's sums go through. */
typedef enum {
    LBI_ACT_NONE = 0, /* z                                                    */
    LBI_ACT_SILU = 1, /* z / (1 + e^-z)                                       */
    LBI_ACT_GELU = 2  /* z (1 + erf(z / sqrt(2))) / 2                         */
} lbi_activation;

/*
 * Matrix product with bias, activation and the residual's addition.
 *
 *   x         [T][K] dt.
 *   weight    [N][K] dt, at row stride ld_weight.
 *   bias      [N] float32, or NULL (= 0).
 *   residual  [T][N] out_dt, or NULL (no addition).
 *   out       OUTPUT [T][N] out_dt: act(z) + residual with z = x W^T + bias,
 *             summed and carried through in float32, rounded once.  May be the
 *             same pointer as residual (with the same stride).
 *   pre       OUTPUT [T][N] dt: z, for the gradient; or NULL (not written).
 *   T >= 0, 1 <= K, N <= LBI_PROJECTION_MAX (else LBI_ERR_SHAPE).
 * dt float32: a value goes into the products as the sum of three bf16 values,
 * of whose nine products six are added in float32: at most 2^-22 of a product is
 * left out.  Below 2^-110 the smaller parts begin to vanish; a value of 3.395e38
 * and more, or an infinity, gives NaN where it is a factor.
 * A NaN or an infinity stays within its row of x, or its row of the weight.
 *   workspace  lbi_projection_workspace_bytes(T, K, N, dt) bytes, 256-byte
 *              aligned (NULL where that is 0): partial sums of calls whose
 *              output is too small to fill the GPU.
 */
size_t lbi_projection_workspace_bytes(int64_t T, int32_t K, int32_t N, lbi_dtype dt);
lbi_status lbi_projection(const void *x, int64_t ld_x, const void *weight, int64_t ld_weight,
                          const float *bias, const void *residual, int64_t ld_residual, void *out,
                          int64_t ld_out, void *pre, int64_t ld_pre, int64_t T, int32_t K,
                          int32_t N, lbi_activation act, lbi_dtype dt, lbi_dtype out_dt,
                          void *workspace, size_t workspace_bytes, lbi_stream_t stream);

/*
 * Gradient of the projection.  (The residual's is dout itself.)
 *
 *   dout       [T][N] out_dt.
 *   pre        [T][N] dt: z of the forward call; ignored for LBI_ACT_NONE.
 *   dx         OUTPUT [T][K] dt: dz W with dz = dout act'(z); or NULL.
 *   dweight    OUTPUT [N][K] dt, at row stride ld_dweight: dz^T x; or NULL.
 *   dbias      OUTPUT [N] float32: the sum over rows of dz; or NULL.
 * dz is formed in float32; as an operand of the two products it is rounded to
 * dt, and float32 products are as above.  All sums are float32.
 *   workspace  lbi_projection_backward_workspace_bytes(...) bytes, 256-byte
 *              aligned (NULL where that is 0).
 */
size_t lbi_projection_backward_workspace_bytes(int64_t T, int32_t K, int32_t N,
                                               lbi_activation act, lbi_dtype dt,
                                               lbi_dtype out_dt);
lbi_status lbi_projection_backward(const void *x, int64_t ld_x, const void *weight,
                                   int64_t ld_weight, const void *dout, int64_t ld_dout,
                                   const void *pre, int64_t ld_pre, void *dx, int64_t ld_dx,
                                   void *dweight, int64_t ld_dweight, float *dbias, int64_t T,
                                   int32_t K, int32_t N, lbi_activation act, lbi_dtype dt,
                                   lbi_dtype out_dt, void *workspace, size_t workspace_bytes,
                                   lbi_stream_t stream);

/* What the forms of the attention read (a HOST struct of DEVICE pointers). */
typedef struct {
    const void *q;           /* [T][H][DK] dt, a token's H DK values dense    */
    int64_t ld_q;
    const void *k;           /* [T][KH][DK] dt                                */
    int64_t ld_k;
    const void *v;           /* [T][KH][DV] dt                                */
    int64_t ld_v;
    const float *log_decay;  /* [H]: logarithm of the factor a with which a
                              * state fades from token to token, 0 (never)
                              * down to -infinity (at once); above 0 or NaN:
                              * the head's results are NaN                    */
    const float *state_in;   /* [sequences or n_slots][H][DK][DV], or NULL
                              * (zeros)                                       */
    const int64_t *offsets;  /* [sequences + 1] DEVICE, or NULL               */
    int64_t T;               /* tokens of all sequences                       */
    int64_t sequences;       /* fewer than 2^32                               */
    int32_t H;               /* heads                                         */
    int32_t KH;              /* heads of k and v: heads h H/KH .. share one;
                              * KH divides H                                  */
    int32_t DK, DV;          /* 1 .. LBI_ATTENTION_MAX_DIM                    */
    float scale;
    lbi_dtype dt;
} lbi_attention_inputs;

/*
 * Linear attention over packed sequences.
 *
 *   o          OUTPUT [T][H][DV] dt, a token's values dense, at row stride ld_o.
 *   state_out  OUTPUT, as state_in: the states after each sequence's last
 *              token; or NULL.
 *   workspace  lbi_linear_attention_workspace_bytes(...) bytes, 256-byte
 *              aligned (NULL where that is 0).  ragged: offsets given.
 * Tokens are taken in chunks: within one by the products of queries and keys,
 * across them by the state, which is float32.  With bf16 tokens the products of
 * queries and keys are rounded to bf16 before they meet the values; a state
 * meets the queries as the sum of two bf16 values (at most 2^-16 away; NaN for a
 * value of 3.395e38 and more, which bf16 does not hold).  A NaN or an infinity in
 * a token reaches no earlier token; one in a state gives a NaN or an infinity in
 * its column, from there on.
 */
size_t lbi_linear_attention_workspace_bytes(int64_t T, int64_t sequences, int32_t H, int32_t KH,
                                            int32_t DK, int32_t DV, int32_t ragged, lbi_dtype dt);
lbi_status lbi_linear_attention(const lbi_attention_inputs *in, void *o, int64_t ld_o,
                                float *state_out, const int32_t *slots, int32_t n_slots,
                                void *workspace, size_t workspace_bytes, lbi_stream_t stream);

/* What lbi_linear_attention_backward writes (a HOST struct of DEVICE pointers). */
typedef struct {
    void *dq;            /* [T][H][DK] dt                                     */
    int64_t ld_dq;
    void *dk;            /* [T][KH][DK] dt                                    */
    int64_t ld_dk;
    void *dv;            /* [T][KH][DV] dt                                    */
    int64_t ld_dv;
    float *dlog_decay;   /* [H], or NULL                                      */
    float *dstate_in;    /* [sequences][H][DK][DV], or NULL                   */
} lbi_attention_gradients;

/*
 * Gradient of lbi_linear_attention (states by sequence, without slots), from
 * the forward's inputs alone: the states are computed again.
 *
 *   dout        [T][H][DV] dt.
 *   dstate_out  [sequences][H][DK][DV] float32: gradient of state_out, or NULL.
 * With bf16 tokens the products over pairs of tokens are rounded to bf16 as
 * operands for dq, dk and dv; states and their gradients enter dq and dk as three
 * bf16 values and dv as two.  dlog_decay is formed from what is not yet rounded.
 */
size_t lbi_linear_attention_backward_workspace_bytes(int64_t T, int64_t sequences, int32_t H,
                                                     int32_t KH, int32_t DK, int32_t DV,
                                                     int32_t ragged, lbi_dtype dt);
lbi_status lbi_linear_attention_backward(const lbi_attention_inputs *in, const void *dout,
                                         int64_t ld_dout, const float *dstate_out,
                                         const lbi_attention_gradients *grads, void *workspace,
                                         size_t workspace_bytes, lbi_stream_t stream);

/*
 * One token for each of in->sequences sequences (in->T must equal it and
 * in->offsets be NULL, else LBI_ERR_SHAPE); in->state_in and state_out are
 * both required and may be the same.  A sequence whose slot is out of range is
 * computed from zeros, and its state is not written.
 */
lbi_status lbi_linear_attention_step(const lbi_attention_inputs *in, void *o, int64_t ld_o,
                                     float *state_out, const int32_t *slots, int32_t n_slots,
                                     lbi_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* LBI_LINEAR_H */
