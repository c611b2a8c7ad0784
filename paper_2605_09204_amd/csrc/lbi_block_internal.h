// Interfaces between the translation units of the region block's operators
// (not part of the public C-ABI in include/lbi_block.h).
#ifndef LBI_BLOCK_INTERNAL_H
#define LBI_BLOCK_INTERNAL_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lbi_block.h"

namespace lbi {

// Workgroups of 256 in a launch, whose work items are fewer than 2^32: more would be refused, or
// their number taken modulo 2^32.
constexpr int64_t kMostGroups = (1 << 24) - 1;

// ---- norm --------------------------------------------------------------------

struct NormArgs {
    const void *x;          // [T][D] token type (gradient: dout)
    const void *residual;   // [T][D] residual type, or NULL (gradient: dresidual)
    const void *s;          // gradient: [T][D] residual type, what was normalised
    const float *weight;    // [D]
    void *out;              // [T][D] token type; bytes for 8-bit forms; gradient: ds
    void *residual_out;     // [T][D] residual type, or NULL
    float *scales;          // 8-bit forms: [T][ngroups]
    float *partial;         // gradient: [blocks][D] partial sums of dweight, or NULL
    int64_t ld_x, ld_residual, ld_s, ld_out, ld_residual_out;
    int64_t T;
    int32_t D;
    float eps;
    int32_t group, ngroups;  // 8-bit forms (group 0: the row)
};
hipError_t launch_rms_norm(const NormArgs &a, bool bf16, bool residual_bf16, hipStream_t stream);
hipError_t launch_rms_norm_q8(const NormArgs &a, bool int8, bool bf16, bool residual_bf16,
                              hipStream_t stream);
// Writes ds and, with a.partial, dweight (out of norm_partial_rows(T, D)
// rows of partial sums).
int64_t norm_partial_rows(int64_t T, int32_t D);
hipError_t launch_rms_norm_backward(const NormArgs &a, float *dweight, bool bf16,
                                    bool residual_bf16, hipStream_t stream);

// ---- convolution -------------------------------------------------------------

struct ConvArgs {
    const void *x;           // [T][D]
    const void *dout;        // gradient: [T][D]
    const float *weight;     // [D][W]
    const float *bias;       // [D] or NULL
    const void *state_in;    // [.][W-1][D] or NULL
    const void *dstate_out;  // gradient: [B][W-1][D] or NULL
    void *out;               // [T][D] (gradient: dx)
    void *state_out;         // [.][W-1][D] or NULL (gradient: dstate_in)
    float *partial;          // gradient: [row blocks][W + 1][D] sums of dweight, dbias
    const int32_t *slots;
    const int64_t *offsets;
    int64_t ld_x, ld_dout, ld_out;
    int64_t T, B;
    int32_t D, W, n_slots;
    bool silu;
};
hipError_t launch_ssm_conv(const ConvArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_ssm_conv_step(const ConvArgs &a, bool bf16, hipStream_t stream);
int64_t conv_partial_rows(int64_t T, int32_t D);
hipError_t launch_ssm_conv_backward(const ConvArgs &a, float *dweight, float *dbias, bool bf16,
                                    hipStream_t stream);

// ---- scan --------------------------------------------------------------------

// How the tokens are cut among workgroups.  per_sequence > 0: every sequence (of
// the same length) into that many ranges of `tokens` tokens; 0: all T rows into
// ranges of `tokens` rows, wherever sequences begin.
struct SsmCut {
    int64_t ranges, tokens;
    int32_t per_sequence;
    int32_t tiles;  // workgroups along the channels, over all groups
    bool joined;    // states pass between ranges
    uint32_t first; // the range that a launch begins with
};
SsmCut ssm_cut(int64_t T, int64_t sequences, int32_t D, int32_t G, bool ragged, double again,
               double launches);

struct SsmArgs {
    lbi_ssm_inputs in;
    void *y;
    int64_t ld_y;
    float *state_out;
    const int32_t *slots;
    int32_t n_slots;
    SsmCut cut;
    // Workspace, for joined ranges.  ends: the state at a range's end (first
    // as if it entered with zeros, then in full); sums: its sum of D_t; starts:
    // the state with which the sequence that leaves the range began; flags:
    // kStarts, kEnds.
    float *ends;    // [ranges][D][N]
    float *sums;    // [ranges][D]
    float *starts;  // [ranges][D][N], with in.state_in only
    int32_t *flags; // [ranges]
    // Gradient.
    const void *dy;
    int64_t ld_dy;
    const float *dstate_out;
    lbi_ssm_gradients out;
    float *marks;      // [ceil(T / step)][D][N] states on the way
    float *mark_sums;  // [ceil(T / step)][D] sums of D_t up to there (joined)
    float *heads;      // [ranges][D][N]: the state's gradient at a range's start (joined)
    float *part_bc;    // [tiles of a group][T][G][N][2]
    float *part_par;   // [ranges][D N + 2 D]: dA, dskip, ddelta_bias
};
enum : int32_t { kStarts = 1, kEnds = 2 };

SsmCut ssm_forward_cut(const lbi_ssm_inputs &in, bool ragged);
hipError_t launch_ssm_scan(const SsmArgs &a, hipStream_t stream);
hipError_t launch_ssm_scan_step(const SsmArgs &a, hipStream_t stream);
SsmCut ssm_backward_cut(const lbi_ssm_inputs &in, bool ragged);
int32_t ssm_backward_step(int32_t N);  // tokens between marks
hipError_t launch_ssm_scan_backward(const SsmArgs &a, hipStream_t stream);

}  // namespace lbi

#endif  // LBI_BLOCK_INTERNAL_H
