// Interfaces between the translation units of the operators in include/lbi_linear.h
// (not part of the public C-ABI).
#ifndef LBI_LINEAR_INTERNAL_H
#define LBI_LINEAR_INTERNAL_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lbi_block_internal.h"
#include "lbi_linear.h"

namespace lbi {

// ---- layer norm (NormArgs)

hipError_t launch_layer_norm(const NormArgs &a, bool bf16, bool residual_bf16, hipStream_t stream);
int64_t layer_norm_partial_rows(int64_t T, int32_t D);  // of [2][D] partial sums
hipError_t launch_layer_norm_backward(const NormArgs &a, float *dweight, float *dbias, bool bf16,
                                      bool residual_bf16, hipStream_t stream);

// ---- projection

// out[m][n] = act(sum_k A(m, k) B(n, k) + bias[n]) + residual[m][n]
struct ProductArgs {
    const void *a, *b;
    int64_t ld_a, ld_b;
    bool a_cols, b_cols;     // stored [k][m], [k][n] instead of [m][k], [n][k]
    int64_t M, K;
    int32_t N;
    const float *bias;       // [N] or NULL
    const void *residual;    // [M][N] of out's type, or NULL
    int64_t ld_residual;
    void *out;
    int64_t ld_out;
    void *pre;               // [M][N] of a's type: before act; or NULL
    int64_t ld_pre;
    lbi_activation act;
    bool bf16, out_bf16;     // a, b and pre; residual and out
    float *partial;          // [splits][M][N], splits > 1 only
    int32_t splits;
    int64_t split;           // values of k of each
    int32_t tile_m, tile_n;  // of a workgroup
};
// Sets the tile, splits and split; returns the floats of partial.
int64_t plan_product(ProductArgs &a);
hipError_t launch_product(const ProductArgs &a, hipStream_t stream);

// dz = dout act'(pre), and the sums of its columns.
struct SlopeArgs {
    const void *dout, *pre;  // pre: NULL for LBI_ACT_NONE
    int64_t ld_dout, ld_pre;
    void *dz;                // [T][N] dense, or NULL
    float *partial;          // [slope_rows(T)][N], or NULL
    int64_t T;
    int32_t N;
    lbi_activation act;
    bool bf16, out_bf16;     // pre and dz; dout
};
int64_t slope_rows(int64_t T);
hipError_t launch_slope(const SlopeArgs &a, float *dbias, hipStream_t stream);

// ---- linear attention

// How the tokens are cut among workgroups: a workgroup walks along `tokens` rows of one head.
// per_sequence > 0: every sequence (of the same length) into that many ranges; 0: all T rows into
// ranges, wherever sequences begin.
struct AttentionCut {
    int64_t ranges, tokens;
    int32_t per_sequence;
    bool joined;  // states pass between ranges
};
AttentionCut attention_cut(const lbi_attention_inputs &in, bool ragged, bool backward);
constexpr int kAttentionTile = 64;  // the unit of a cut's tokens
// States that the gradient keeps of a range and head, one of them for scratch.
int64_t attention_marks(const lbi_attention_inputs &in, const AttentionCut &cut);

struct AttentionArgs {
    lbi_attention_inputs in;
    void *o;
    int64_t ld_o;
    float *state_out;
    const int32_t *slots;
    int32_t n_slots;
    AttentionCut cut;
    // Workspace, for joined ranges: the state at a range's end (first as if it entered with zeros,
    // then in full), the gradient of the state at a range's start, and kWhole, kPart or 0 (no
    // sequence passes the range's end, or start).
    float *ends, *heads;             // [ranges][H][DK][DV]
    // States in place: those with which sequences begin that end in another range, whose workgroup
    // writes their slots.
    float *starts;                   // [ranges][H][DK][DV], or NULL
    int32_t *end_flags, *head_flags; // [ranges]
    // Gradient.
    const void *dout;
    int64_t ld_dout;
    const float *dstate_out;
    lbi_attention_gradients out;
    float *marks;          // [ranges][H][attention_marks][DK][DV]: states on the way, less
                           // what enters the range
    float *part_k, *part_v; // [T][H][DK or DV]: shared heads' gradients by head, KH < H only
    float *part_decay;     // [ranges][H]
};
enum : int32_t { kPart = 1, kWhole = 2 };

hipError_t launch_linear_attention(const AttentionArgs &a, hipStream_t stream);
hipError_t launch_linear_attention_step(const AttentionArgs &a, hipStream_t stream);
hipError_t launch_linear_attention_backward(const AttentionArgs &a, hipStream_t stream);
// The states at the ranges' ends and, for both, their gradients at the ranges' starts; with marks,
// also the states before tiles of mark_rows tokens, as far as the range they are in adds to them.
hipError_t launch_attention_ends(const AttentionArgs &a, bool both, int mark_rows, int marks,
                                 hipStream_t stream);
// States (or their gradients) of sequences without tokens.
hipError_t launch_attention_empty(const AttentionArgs &a, bool backward, hipStream_t stream);

}  // namespace lbi

#endif  // LBI_LINEAR_INTERNAL_H
