// C entry points of the region block's operators (include/lbi_block.h): argument
// checks, workspace layout and launches.
#include "lbi_block_checks.hpp"

using namespace lbi;

namespace {

// ---- norm

lbi_status norm_forward(const NormArgs &a, size_t out_element, lbi_dtype dt, lbi_dtype rdt)
{
    if (a.T == 0)
        return LBI_OK;
    if (!a.x || !a.weight || !a.out || (a.residual_out && !a.residual))
        return LBI_ERR_NULL;
    const Tensor x = tokens(a.x, a.T, a.D, a.ld_x, size_of(dt));
    const Tensor res = tokens(a.residual, a.T, a.D, a.ld_residual, size_of(rdt));
    const Tensor w = dense(a.weight, 1, a.D, 4);
    const Tensor out = tokens(a.out, a.T, a.D, a.ld_out, out_element);
    const Tensor total = tokens(a.residual_out, a.T, a.D, a.ld_residual_out, size_of(rdt));
    const Tensor scales = dense(a.scales, a.T, a.ngroups, 4);
    return check_tensors({x, res, w}, {out, total, scales}, &total, &res);
}

// ---- scan

bool bad_scan_shape(int64_t T, int64_t sequences, int32_t D, int32_t N, int32_t G, bool ragged)
{
    if (T < 0 || T > kMostRows || sequences < 0 || sequences > kMostRows || D < 1 ||
        D > LBI_SSM_MAX_D || N < 1 || N > LBI_SSM_MAX_N || G < 1 || D % G != 0)
        return true;
    return sequences == 0 ? T != 0 : !ragged && T % sequences != 0;
}

lbi_status check_scan_inputs(const lbi_ssm_inputs *in)
{
    if (!in)
        return LBI_ERR_NULL;
    if (!known(in->dt))
        return LBI_ERR_DTYPE;
    if (bad_scan_shape(in->T, in->sequences, in->D, in->N, in->G, in->offsets != nullptr))
        return LBI_ERR_SHAPE;
    if (in->sequences > 0 && !in->A)
        return LBI_ERR_NULL;
    if (in->T > 0 && (!in->u || !in->delta || !in->B || !in->C))
        return LBI_ERR_NULL;
    return LBI_OK;
}

struct ScanTensors {
    Tensor u, delta, z, B, C, A, skip, bias, state, offsets;
    ScanTensors(const lbi_ssm_inputs &in, int64_t state_rows)
    {
        const size_t e = size_of(in.dt);
        const int64_t gn = (int64_t)in.G * in.N;
        u = tokens(in.u, in.T, in.D, in.ld_u, e);
        delta = tokens(in.delta, in.T, in.D, in.ld_delta, e);
        z = tokens(in.z, in.T, in.D, in.ld_z, e);
        B = tokens(in.B, in.T, gn, in.ld_B, e);
        C = tokens(in.C, in.T, gn, in.ld_C, e);
        A = dense(in.A, in.D, in.N, 4);
        skip = dense(in.skip, 1, in.D, 4);
        bias = dense(in.delta_bias, 1, in.D, 4);
        state = dense(in.state_in, state_rows, (int64_t)in.D * in.N, 4);
        offsets = dense(in.offsets, 1, in.sequences + 1, 8);
    }
};

// The rows of a tile or piece are addressed by 32-bit distances in bytes.
bool too_wide(std::initializer_list<int64_t> strides)
{
    for (int64_t ld : strides)
        if (ld > LBI_SSM_MAX_LD)
            return true;
    return false;
}

bool too_many_ranges(const SsmCut &c) { return c.ranges > UINT32_MAX; }

size_t scan_layout(SsmArgs &a, void *workspace)
{
    Layout l{(char *)workspace};
    if (a.cut.joined) {
        const int64_t dN = (int64_t)a.in.D * a.in.N;
        a.ends = l.take<float>(a.cut.ranges * dN);
        a.sums = l.take<float>(a.cut.ranges * a.in.D);
        a.starts = l.take<float>(a.cut.ranges * dN);
        a.flags = l.take<int32_t>(a.cut.ranges);
    }
    return l.used;
}

}  // namespace

extern "C" {

lbi_status lbi_rms_norm(const void *x, int64_t ld_x, const void *residual, int64_t ld_residual,
                        const float *weight, void *out, int64_t ld_out, void *residual_out,
                        int64_t ld_residual_out, int64_t T, int32_t D, float eps, lbi_dtype dt,
                        lbi_dtype residual_dt, lbi_stream_t stream)
{
    if (!known(dt) || !known(residual_dt))
        return LBI_ERR_DTYPE;
    if (bad_norm_shape(T, D, eps))
        return LBI_ERR_SHAPE;
    NormArgs a = {};
    a.x = x; a.ld_x = ld_x;
    a.residual = residual; a.ld_residual = ld_residual;
    a.weight = weight;
    a.out = out; a.ld_out = ld_out;
    a.residual_out = residual_out; a.ld_residual_out = ld_residual_out;
    a.T = T; a.D = D; a.eps = eps;
    const lbi_status st = norm_forward(a, size_of(dt), dt, residual_dt);
    if (st != LBI_OK || T == 0)
        return st;
    return status_of(launch_rms_norm(a, dt == LBI_BF16, residual_dt == LBI_BF16,
                                     (hipStream_t)stream));
}

lbi_status lbi_rms_norm_q8(const void *x, int64_t ld_x, const void *residual,
                           int64_t ld_residual, const float *weight, void *q, int64_t ld_q,
                           float *scales, void *residual_out, int64_t ld_residual_out, int64_t T,
                           int32_t D, float eps, int32_t group, lbi_q8_format format,
                           lbi_dtype dt, lbi_dtype residual_dt, lbi_stream_t stream)
{
    if (!known(dt) || !known(residual_dt) || (format != LBI_Q8_E4M3 && format != LBI_Q8_INT8))
        return LBI_ERR_DTYPE;
    if (bad_norm_shape(T, D, eps) || (group != 0 && group != 32 && group != 64 && group != 128))
        return LBI_ERR_SHAPE;
    NormArgs a = {};
    a.x = x; a.ld_x = ld_x;
    a.residual = residual; a.ld_residual = ld_residual;
    a.weight = weight;
    a.out = q; a.ld_out = ld_q;
    a.scales = scales;
    a.residual_out = residual_out; a.ld_residual_out = ld_residual_out;
    a.T = T; a.D = D; a.eps = eps;
    a.group = group;
    a.ngroups = group ? (D + group - 1) / group : 1;
    if (T > 0 && !scales)
        return LBI_ERR_NULL;
    const lbi_status st = norm_forward(a, 1, dt, residual_dt);
    if (st != LBI_OK || T == 0)
        return st;
    return status_of(launch_rms_norm_q8(a, format == LBI_Q8_INT8, dt == LBI_BF16,
                                        residual_dt == LBI_BF16, (hipStream_t)stream));
}

size_t lbi_rms_norm_backward_workspace_bytes(int64_t T, int32_t D)
{
    if (bad_norm_shape(T, D, 0.f) || T == 0)
        return 0;
    return (size_t)norm_partial_rows(T, D) * D * sizeof(float);
}

lbi_status lbi_rms_norm_backward(const void *dout, int64_t ld_dout, const void *s, int64_t ld_s,
                                 const float *weight, const void *dresidual,
                                 int64_t ld_dresidual, void *ds, int64_t ld_ds, float *dweight,
                                 int64_t T, int32_t D, float eps, lbi_dtype dt,
                                 lbi_dtype residual_dt, void *workspace, size_t workspace_bytes,
                                 lbi_stream_t stream)
{
    if (!known(dt) || !known(residual_dt))
        return LBI_ERR_DTYPE;
    if (bad_norm_shape(T, D, eps))
        return LBI_ERR_SHAPE;
    if (T > 0 && (!dout || !s || !weight || !ds))
        return LBI_ERR_NULL;
    const size_t need = dweight ? lbi_rms_norm_backward_workspace_bytes(T, D) : 0;
    const size_t re = size_of(residual_dt);
    const Tensor d = tokens(ds, T, D, ld_ds, re), dr = tokens(dresidual, T, D, ld_dresidual, re);
    lbi_status st = check_workspace(workspace, workspace_bytes, need);
    if (st != LBI_OK)
        return st;
    st = check_tensors({tokens(dout, T, D, ld_dout, size_of(dt)), tokens(s, T, D, ld_s, re),
                        dense(weight, 1, D, 4), dr},
                       {d, dense(dweight, 1, D, 4),
                        dense(need ? workspace : nullptr, 1, (int64_t)need, 1)},
                       &d, &dr);
    if (st != LBI_OK)
        return st;
    NormArgs a = {};
    a.x = dout; a.ld_x = ld_dout;
    a.s = s; a.ld_s = ld_s;
    a.residual = dresidual; a.ld_residual = ld_dresidual;
    a.weight = weight;
    a.out = ds; a.ld_out = ld_ds;
    a.partial = dweight ? (float *)workspace : nullptr;
    a.T = T; a.D = D; a.eps = eps;
    return status_of(launch_rms_norm_backward(a, dweight, dt == LBI_BF16,
                                              residual_dt == LBI_BF16, (hipStream_t)stream));
}

static bool bad_conv_shape(int64_t T, int64_t B, int32_t D, int32_t W, bool ragged)
{
    if (T < 0 || T > kMostRows || B < 0 || B > kMostRows || D < 1 || D > LBI_SSM_MAX_D || W < 2 ||
        W > LBI_CONV_MAX_W)
        return true;
    return B == 0 ? T != 0 : !ragged && T % B != 0;
}

lbi_status lbi_ssm_conv(const void *x, int64_t ld_x, const float *weight, const float *bias,
                        void *out, int64_t ld_out, const void *state_in, void *state_out,
                        const int32_t *slots, int32_t n_slots, const int64_t *offsets, int64_t T,
                        int64_t B, int32_t D, int32_t W, int32_t silu, lbi_dtype dt,
                        lbi_stream_t stream)
{
    if (!known(dt))
        return LBI_ERR_DTYPE;
    if (bad_conv_shape(T, B, D, W, offsets != nullptr) || (slots && n_slots < 0) ||
        too_wide({ld_x, ld_out}))
        return LBI_ERR_SHAPE;
    if (B == 0)
        return LBI_OK;
    if (!weight || (T > 0 && (!x || !out)))
        return LBI_ERR_NULL;
    const size_t e = size_of(dt);
    const int64_t rows = slots ? n_slots : B;
    const Tensor in = dense(state_in, rows, (int64_t)(W - 1) * D, e);
    const Tensor to = dense(state_out, rows, (int64_t)(W - 1) * D, e);
    const lbi_status st = check_tensors(
        {tokens(x, T, D, ld_x, e), dense(weight, D, W, 4), dense(bias, 1, D, 4), in,
         dense(slots, 1, B, 4), dense(offsets, 1, B + 1, 8)},
        {tokens(out, T, D, ld_out, e), to}, &to, &in);
    if (st != LBI_OK)
        return st;
    ConvArgs a = {};
    a.x = x; a.ld_x = ld_x;
    a.weight = weight; a.bias = bias;
    a.out = out; a.ld_out = ld_out;
    a.state_in = state_in; a.state_out = state_out;
    a.slots = slots; a.n_slots = n_slots;
    a.offsets = offsets;
    a.T = T; a.B = B; a.D = D; a.W = W; a.silu = silu != 0;
    return status_of(launch_ssm_conv(a, dt == LBI_BF16, (hipStream_t)stream));
}

size_t lbi_ssm_conv_backward_workspace_bytes(int64_t T, int32_t D, int32_t W)
{
    if (T <= 0 || bad_conv_shape(T, T, D, W, true))
        return 0;
    return (size_t)conv_partial_rows(T, D) * (W + 1) * D * sizeof(float);
}

lbi_status lbi_ssm_conv_backward(const void *x, int64_t ld_x, const float *weight,
                                 const float *bias, const void *dout, int64_t ld_dout,
                                 const void *state_in, const void *dstate_out, void *dx,
                                 int64_t ld_dx, float *dweight, float *dbias, void *dstate_in,
                                 const int64_t *offsets, int64_t T, int64_t B, int32_t D,
                                 int32_t W, int32_t silu, lbi_dtype dt, void *workspace,
                                 size_t workspace_bytes, lbi_stream_t stream)
{
    if (!known(dt))
        return LBI_ERR_DTYPE;
    if (bad_conv_shape(T, B, D, W, offsets != nullptr) || too_wide({ld_x, ld_dout, ld_dx}))
        return LBI_ERR_SHAPE;
    if (!weight || !dweight || (T > 0 && (!x || !dout || !dx)))
        return LBI_ERR_NULL;
    const size_t need = lbi_ssm_conv_backward_workspace_bytes(T, D, W);
    lbi_status st = check_workspace(workspace, workspace_bytes, need);
    if (st != LBI_OK)
        return st;
    const size_t e = size_of(dt);
    const int64_t state = (int64_t)(W - 1) * D;
    st = check_tensors({tokens(x, T, D, ld_x, e), dense(weight, D, W, 4), dense(bias, 1, D, 4),
                        tokens(dout, T, D, ld_dout, e), dense(state_in, B, state, e),
                        dense(dstate_out, B, state, e), dense(offsets, 1, B + 1, 8)},
                       {tokens(dx, T, D, ld_dx, e), dense(dweight, D, W, 4), dense(dbias, 1, D, 4),
                        dense(dstate_in, B, state, e),
                        dense(need ? workspace : nullptr, 1, (int64_t)need, 1)});
    if (st != LBI_OK)
        return st;
    ConvArgs a = {};
    a.x = x; a.ld_x = ld_x;
    a.weight = weight; a.bias = bias;
    a.dout = dout; a.ld_dout = ld_dout;
    a.state_in = state_in; a.dstate_out = dstate_out;
    a.out = dx; a.ld_out = ld_dx;
    a.state_out = dstate_in;
    a.offsets = offsets;
    a.T = T; a.B = B; a.D = D; a.W = W; a.silu = silu != 0;
    a.partial = (float *)workspace;
    return status_of(launch_ssm_conv_backward(a, dweight, dbias, dt == LBI_BF16,
                                              (hipStream_t)stream));
}

lbi_status lbi_ssm_conv_step(const void *x, int64_t ld_x, const float *weight, const float *bias,
                             void *out, int64_t ld_out, const void *state_in, void *state_out,
                             const int32_t *slots, int32_t n_slots, int64_t n, int32_t D,
                             int32_t W, int32_t silu, lbi_dtype dt, lbi_stream_t stream)
{
    if (!known(dt))
        return LBI_ERR_DTYPE;
    if (bad_conv_shape(n, n, D, W, true) || (slots && n_slots < 0))
        return LBI_ERR_SHAPE;
    if (n == 0)
        return LBI_OK;
    if (!x || !weight || !out || !state_in || !state_out)
        return LBI_ERR_NULL;
    const size_t e = size_of(dt);
    const int64_t rows = slots ? n_slots : n;
    const Tensor in = dense(state_in, rows, (int64_t)(W - 1) * D, e);
    const Tensor to = dense(state_out, rows, (int64_t)(W - 1) * D, e);
    const lbi_status st = check_tensors({tokens(x, n, D, ld_x, e), dense(weight, D, W, 4),
                                         dense(bias, 1, D, 4), in, dense(slots, 1, n, 4)},
                                        {tokens(out, n, D, ld_out, e), to}, &to, &in);
    if (st != LBI_OK)
        return st;
    ConvArgs a = {};
    a.x = x; a.ld_x = ld_x;
    a.weight = weight; a.bias = bias;
    a.out = out; a.ld_out = ld_out;
    a.state_in = state_in; a.state_out = state_out;
    a.slots = slots; a.n_slots = n_slots;
    a.T = n; a.B = n; a.D = D; a.W = W; a.silu = silu != 0;
    return status_of(launch_ssm_conv_step(a, dt == LBI_BF16, (hipStream_t)stream));
}

size_t lbi_ssm_scan_workspace_bytes(int64_t T, int64_t sequences, int32_t D, int32_t N,
                                    int32_t G, int32_t ragged)
{
    if (bad_scan_shape(T, sequences, D, N, G, ragged != 0) || sequences == 0)
        return 0;
    SsmArgs a = {};
    a.in.T = T; a.in.sequences = sequences;
    a.in.D = D; a.in.N = N; a.in.G = G;
    a.cut = ssm_forward_cut(a.in, ragged != 0);
    return scan_layout(a, nullptr);
}

lbi_status lbi_ssm_scan(const lbi_ssm_inputs *in, void *y, int64_t ld_y, float *state_out,
                        const int32_t *slots, int32_t n_slots, void *workspace,
                        size_t workspace_bytes, lbi_stream_t stream)
{
    lbi_status st = check_scan_inputs(in);
    if (st != LBI_OK)
        return st;
    if (slots && n_slots < 0)
        return LBI_ERR_SHAPE;
    if (in->sequences == 0)
        return LBI_OK;
    if (in->T > 0 && !y)
        return LBI_ERR_NULL;
    SsmArgs a = {};
    a.in = *in;
    a.y = y; a.ld_y = ld_y;
    a.state_out = state_out;
    a.slots = slots; a.n_slots = n_slots;
    a.cut = ssm_forward_cut(*in, in->offsets != nullptr);
    if (too_many_ranges(a.cut) || too_wide({in->ld_u, in->ld_delta, in->z ? in->ld_z : 0, in->ld_B,
                                            in->ld_C, ld_y}))
        return LBI_ERR_SHAPE;
    const size_t need = scan_layout(a, workspace);
    st = check_workspace(workspace, workspace_bytes, need);
    if (st != LBI_OK)
        return st;
    const int64_t rows = slots ? n_slots : in->sequences;
    const ScanTensors t(*in, rows);
    const Tensor to = dense(state_out, rows, (int64_t)in->D * in->N, 4);
    st = check_tensors({t.u, t.delta, t.z, t.B, t.C, t.A, t.skip, t.bias, t.state, t.offsets,
                        dense(slots, 1, in->sequences, 4)},
                       {tokens(y, in->T, in->D, ld_y, size_of(in->dt)), to,
                        dense(need ? workspace : nullptr, 1, (int64_t)need, 1)},
                       &to, &t.state);
    if (st != LBI_OK)
        return st;
    return status_of(launch_ssm_scan(a, (hipStream_t)stream));
}

static size_t backward_layout(SsmArgs &a, void *workspace)
{
    Layout l{(char *)workspace};
    const int64_t T = a.in.T, D = a.in.D, N = a.in.N, G = a.in.G, dN = D * N;
    if (T == 0)
        return 0;
    const int64_t marks = (T + ssm_backward_step(a.in.N) - 1) / ssm_backward_step(a.in.N);
    a.marks = l.take<float>(marks * dN);
    if (a.cut.joined) {
        a.mark_sums = l.take<float>(marks * D);
        a.ends = l.take<float>(a.cut.ranges * dN);
        a.sums = l.take<float>(a.cut.ranges * D);
        a.heads = l.take<float>(a.cut.ranges * dN);
        a.flags = l.take<int32_t>(a.cut.ranges);
    }
    a.part_bc = l.take<float>(a.cut.tiles / G * T * G * N * 2);
    a.part_par = l.take<float>(a.cut.ranges * (dN + 2 * D));
    return l.used;
}

size_t lbi_ssm_scan_backward_workspace_bytes(int64_t T, int64_t sequences, int32_t D, int32_t N,
                                             int32_t G, int32_t ragged)
{
    if (bad_scan_shape(T, sequences, D, N, G, ragged != 0) || sequences == 0)
        return 0;
    SsmArgs a = {};
    a.in.T = T; a.in.sequences = sequences;
    a.in.D = D; a.in.N = N; a.in.G = G;
    a.cut = ssm_backward_cut(a.in, ragged != 0);
    return backward_layout(a, nullptr);
}

lbi_status lbi_ssm_scan_backward(const lbi_ssm_inputs *in, const void *dy, int64_t ld_dy,
                                 const float *dstate_out, const lbi_ssm_gradients *grads,
                                 void *workspace, size_t workspace_bytes, lbi_stream_t stream)
{
    lbi_status st = check_scan_inputs(in);
    if (st != LBI_OK)
        return st;
    if (!grads || !grads->dA || !in->A ||
        (in->T > 0 && (!dy || !grads->du || !grads->ddelta || !grads->dB || !grads->dC ||
                       (in->z && !grads->dz))))
        return LBI_ERR_NULL;
    SsmArgs a = {};
    a.in = *in;
    a.dy = dy; a.ld_dy = ld_dy;
    a.dstate_out = dstate_out;
    a.out = *grads;
    if (!in->z)
        a.out.dz = nullptr;
    a.cut = ssm_backward_cut(*in, in->offsets != nullptr);
    const size_t need = backward_layout(a, workspace);
    if (too_many_ranges(a.cut) ||
        too_wide({in->ld_u, in->ld_delta, in->z ? in->ld_z : 0, in->ld_B, in->ld_C, ld_dy,
                  grads->ld_du, grads->ld_ddelta, in->z ? grads->ld_dz : 0, grads->ld_dB,
                  grads->ld_dC}))
        return LBI_ERR_SHAPE;
    st = check_workspace(workspace, workspace_bytes, need);
    if (st != LBI_OK)
        return st;
    const ScanTensors t(*in, in->sequences);
    const size_t e = size_of(in->dt);
    const int64_t T = in->T, D = in->D, gn = (int64_t)in->G * in->N, dN = D * in->N;
    st = check_tensors({t.u, t.delta, t.z, t.B, t.C, t.A, t.skip, t.bias, t.state, t.offsets,
                        tokens(dy, T, D, ld_dy, e), dense(dstate_out, in->sequences, dN, 4)},
                       {tokens(a.out.du, T, D, a.out.ld_du, e),
                        tokens(a.out.ddelta, T, D, a.out.ld_ddelta, e),
                        tokens(a.out.dz, T, D, a.out.ld_dz, e),
                        tokens(a.out.dB, T, gn, a.out.ld_dB, e),
                        tokens(a.out.dC, T, gn, a.out.ld_dC, e), dense(a.out.dA, D, in->N, 4),
                        dense(a.out.dskip, 1, D, 4), dense(a.out.ddelta_bias, 1, D, 4),
                        dense(a.out.dstate_in, in->sequences, dN, 4),
                        dense(need ? workspace : nullptr, 1, (int64_t)need, 1)});
    if (st != LBI_OK)
        return st;
    return status_of(launch_ssm_scan_backward(a, (hipStream_t)stream));
}

lbi_status lbi_ssm_scan_step(const lbi_ssm_inputs *in, void *y, int64_t ld_y, float *state_out,
                             const int32_t *slots, int32_t n_slots, lbi_stream_t stream)
{
    lbi_status st = check_scan_inputs(in);
    if (st != LBI_OK)
        return st;
    if (in->T != in->sequences || in->offsets || (slots && n_slots < 0))
        return LBI_ERR_SHAPE;
    if (in->sequences == 0)
        return LBI_OK;
    if (!y || !in->state_in || !state_out)
        return LBI_ERR_NULL;
    const int64_t rows = slots ? n_slots : in->sequences;
    const ScanTensors t(*in, rows);
    const Tensor to = dense(state_out, rows, (int64_t)in->D * in->N, 4);
    st = check_tensors({t.u, t.delta, t.z, t.B, t.C, t.A, t.skip, t.bias, t.state,
                        dense(slots, 1, in->sequences, 4)},
                       {tokens(y, in->T, in->D, ld_y, size_of(in->dt)), to}, &to, &t.state);
    if (st != LBI_OK)
        return st;
    SsmArgs a = {};
    a.in = *in;
    a.y = y; a.ld_y = ld_y;
    a.state_out = state_out;
    a.slots = slots; a.n_slots = n_slots;
    return status_of(launch_ssm_scan_step(a, (hipStream_t)stream));
}

}  // extern "C"
