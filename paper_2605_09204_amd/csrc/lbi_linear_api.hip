// C entry points of the operators in include/lbi_linear.h: argument checks, workspace layout and
// launches.
#include "lbi_block_checks.hpp"
#include "lbi_linear_internal.h"

using namespace lbi;

namespace {

// ---- layer norm

lbi_status layer_norm_tensors(const NormArgs &a, lbi_dtype dt, lbi_dtype rdt)
{
    if (a.T == 0)
        return LBI_OK;
    if (!a.x || !a.out || (a.residual_out && !a.residual))
        return LBI_ERR_NULL;
    const Tensor res = tokens(a.residual, a.T, a.D, a.ld_residual, size_of(rdt));
    const Tensor total = tokens(a.residual_out, a.T, a.D, a.ld_residual_out, size_of(rdt));
    return check_tensors({tokens(a.x, a.T, a.D, a.ld_x, size_of(dt)), res, dense(a.weight, 1, a.D, 4),
                          dense(a.bias, 1, a.D, 4)},
                         {tokens(a.out, a.T, a.D, a.ld_out, size_of(dt)), total}, &total, &res);
}

// ---- projection

bool bad_projection_shape(int64_t T, int32_t K, int32_t N)
{
    return T < 0 || T > kMostRows || K < 1 || K > LBI_PROJECTION_MAX || N < 1 ||
           N > LBI_PROJECTION_MAX;
}
bool known_act(lbi_activation act)
{
    return act == LBI_ACT_NONE || act == LBI_ACT_SILU || act == LBI_ACT_GELU;
}

ProductArgs forward_product(int64_t T, int32_t K, int32_t N, lbi_dtype dt)
{
    ProductArgs a = {};
    a.M = T; a.K = K; a.N = N;
    a.bf16 = dt == LBI_BF16;
    return a;
}

// The gradient's steps: dz (where dout is not it already) and its sums, dx, dweight.
struct ProjectionGradient {
    SlopeArgs slope = {};
    ProductArgs dx = {}, dweight = {};

    ProjectionGradient(int64_t T, int32_t K, int32_t N, lbi_activation act, lbi_dtype dt,
                       lbi_dtype out_dt)
    {
        slope.T = T; slope.N = N;
        slope.act = act;
        slope.bf16 = dt == LBI_BF16;
        slope.out_bf16 = out_dt == LBI_BF16;
        dx.M = T; dx.K = N; dx.N = K;
        dx.b_cols = true;
        dx.bf16 = dx.out_bf16 = slope.bf16;
        dweight.M = N; dweight.K = T; dweight.N = K;
        dweight.a_cols = dweight.b_cols = true;
        dweight.bf16 = dweight.out_bf16 = slope.bf16;
    }
    bool separate() const { return slope.act != LBI_ACT_NONE || slope.bf16 != slope.out_bf16; }
    size_t layout(void *workspace)
    {
        if (slope.T == 0)
            return 0;
        Layout l{(char *)workspace};
        if (separate()) {
            const int64_t n = slope.T * slope.N;
            slope.dz = slope.bf16 ? (void *)l.take<uint16_t>(n) : (void *)l.take<float>(n);
        }
        slope.partial = l.take<float>(slope_rows(slope.T) * slope.N);
        // the two products come one after the other
        const int64_t px = plan_product(dx), pw = plan_product(dweight);
        const int64_t p = px > pw ? px : pw;
        if (p > 0)
            dx.partial = dweight.partial = l.take<float>(p);
        return l.used;
    }
};

// ---- attention

bool bad_attention_shape(int64_t T, int64_t sequences, int32_t H, int32_t KH, int32_t DK,
                         int32_t DV, bool ragged)
{
    if (T < 0 || T > kMostRows || sequences < 0 || sequences > (int64_t)UINT32_MAX || H < 1 ||
        H > LBI_ATTENTION_MAX_H || KH < 1 || H % KH != 0 || DK < 1 || DK > LBI_ATTENTION_MAX_DIM ||
        DV < 1 || DV > LBI_ATTENTION_MAX_DIM)
        return true;
    return sequences == 0 ? T != 0 : !ragged && T % sequences != 0;
}

// The rows of a tile are addressed by 32-bit distances in bytes.
bool too_wide(std::initializer_list<int64_t> strides)
{
    for (int64_t ld : strides)
        if (ld > LBI_ATTENTION_MAX_LD)
            return true;
    return false;
}

lbi_status check_attention_inputs(const lbi_attention_inputs *in)
{
    if (!in)
        return LBI_ERR_NULL;
    if (!known(in->dt))
        return LBI_ERR_DTYPE;
    if (bad_attention_shape(in->T, in->sequences, in->H, in->KH, in->DK, in->DV,
                            in->offsets != nullptr))
        return LBI_ERR_SHAPE;
    if (in->sequences > 0 && !in->log_decay)
        return LBI_ERR_NULL;
    if (in->T > 0 && (!in->q || !in->k || !in->v))
        return LBI_ERR_NULL;
    if (too_wide({in->ld_q, in->ld_k, in->ld_v}))
        return LBI_ERR_SHAPE;
    return LBI_OK;
}

struct AttentionTensors {
    Tensor q, k, v, decay, state, offsets;
    AttentionTensors(const lbi_attention_inputs &in, int64_t state_rows)
    {
        const size_t e = size_of(in.dt);
        q = tokens(in.q, in.T, (int64_t)in.H * in.DK, in.ld_q, e);
        k = tokens(in.k, in.T, (int64_t)in.KH * in.DK, in.ld_k, e);
        v = tokens(in.v, in.T, (int64_t)in.KH * in.DV, in.ld_v, e);
        decay = dense(in.log_decay, 1, in.H, 4);
        state = dense(in.state_in, state_rows, (int64_t)in.H * in.DK * in.DV, 4);
        offsets = dense(in.offsets, 1, in.sequences + 1, 8);
    }
};

lbi_attention_inputs attention_sizes(int64_t T, int64_t sequences, int32_t H, int32_t KH,
                                     int32_t DK, int32_t DV, lbi_dtype dt)
{
    lbi_attention_inputs in = {};
    in.T = T; in.sequences = sequences;
    in.H = H; in.KH = KH;
    in.DK = DK; in.DV = DV;
    in.dt = dt;
    return in;
}

size_t attention_layout(AttentionArgs &a, void *workspace)
{
    Layout l{(char *)workspace};
    if (a.cut.joined) {
        const int64_t n = a.cut.ranges * a.in.H * a.in.DK * a.in.DV;
        a.ends = l.take<float>(n);
        a.starts = l.take<float>(n);
        a.end_flags = l.take<int32_t>(a.cut.ranges);
    }
    return l.used;
}

size_t attention_backward_layout(AttentionArgs &a, void *workspace)
{
    const int64_t T = a.in.T, H = a.in.H, size = (int64_t)a.in.DK * a.in.DV;
    if (T == 0)
        return 0;
    Layout l{(char *)workspace};
    if (a.cut.joined) {
        a.ends = l.take<float>(a.cut.ranges * H * size);
        a.heads = l.take<float>(a.cut.ranges * H * size);
        a.end_flags = l.take<int32_t>(a.cut.ranges);
        a.head_flags = l.take<int32_t>(a.cut.ranges);
    }
    a.marks = l.take<float>(a.cut.ranges * H * attention_marks(a.in, a.cut) * size);
    if (a.in.KH < a.in.H) {
        a.part_k = l.take<float>(T * H * a.in.DK);
        a.part_v = l.take<float>(T * H * a.in.DV);
    }
    a.part_decay = l.take<float>(a.cut.ranges * H);
    return l.used;
}

}  // namespace

extern "C" {

lbi_status lbi_layer_norm(const void *x, int64_t ld_x, const void *residual, int64_t ld_residual,
                          const float *weight, const float *bias, void *out, int64_t ld_out,
                          void *residual_out, int64_t ld_residual_out, int64_t T, int32_t D,
                          float eps, lbi_dtype dt, lbi_dtype residual_dt, lbi_stream_t stream)
{
    if (!known(dt) || !known(residual_dt))
        return LBI_ERR_DTYPE;
    if (bad_norm_shape(T, D, eps))
        return LBI_ERR_SHAPE;
    NormArgs a = {};
    a.x = x; a.ld_x = ld_x;
    a.residual = residual; a.ld_residual = ld_residual;
    a.weight = weight;
    a.bias = bias;
    a.out = out; a.ld_out = ld_out;
    a.residual_out = residual_out; a.ld_residual_out = ld_residual_out;
    a.T = T; a.D = D; a.eps = eps;
    const lbi_status st = layer_norm_tensors(a, dt, residual_dt);
    if (st != LBI_OK || T == 0)
        return st;
    return status_of(launch_layer_norm(a, dt == LBI_BF16, residual_dt == LBI_BF16,
                                       (hipStream_t)stream));
}

size_t lbi_layer_norm_backward_workspace_bytes(int64_t T, int32_t D)
{
    if (bad_norm_shape(T, D, 0.f) || T == 0)
        return 0;
    return (size_t)layer_norm_partial_rows(T, D) * 2 * D * sizeof(float);
}

lbi_status lbi_layer_norm_backward(const void *dout, int64_t ld_dout, const void *s, int64_t ld_s,
                                   const float *weight, const void *dresidual,
                                   int64_t ld_dresidual, void *ds, int64_t ld_ds, float *dweight,
                                   float *dbias, int64_t T, int32_t D, float eps, lbi_dtype dt,
                                   lbi_dtype residual_dt, void *workspace, size_t workspace_bytes,
                                   lbi_stream_t stream)
{
    if (!known(dt) || !known(residual_dt))
        return LBI_ERR_DTYPE;
    if (bad_norm_shape(T, D, eps))
        return LBI_ERR_SHAPE;
    if (T > 0 && (!dout || !s || !ds))
        return LBI_ERR_NULL;
    const bool sums = dweight || dbias;
    const size_t need = sums ? lbi_layer_norm_backward_workspace_bytes(T, D) : 0;
    const size_t re = size_of(residual_dt);
    const Tensor d = tokens(ds, T, D, ld_ds, re), dr = tokens(dresidual, T, D, ld_dresidual, re);
    lbi_status st = check_workspace(workspace, workspace_bytes, need);
    if (st != LBI_OK)
        return st;
    st = check_tensors({tokens(dout, T, D, ld_dout, size_of(dt)), tokens(s, T, D, ld_s, re),
                        dense(weight, 1, D, 4), dr},
                       {d, dense(dweight, 1, D, 4), dense(dbias, 1, D, 4),
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
    a.partial = sums ? (float *)workspace : nullptr;
    a.T = T; a.D = D; a.eps = eps;
    return status_of(launch_layer_norm_backward(a, dweight, dbias, dt == LBI_BF16,
                                                residual_dt == LBI_BF16, (hipStream_t)stream));
}

size_t lbi_projection_workspace_bytes(int64_t T, int32_t K, int32_t N, lbi_dtype dt)
{
    if (!known(dt) || bad_projection_shape(T, K, N) || T == 0)
        return 0;
    ProductArgs a = forward_product(T, K, N, dt);
    return (size_t)plan_product(a) * sizeof(float);
}

lbi_status lbi_projection(const void *x, int64_t ld_x, const void *weight, int64_t ld_weight,
                          const float *bias, const void *residual, int64_t ld_residual, void *out,
                          int64_t ld_out, void *pre, int64_t ld_pre, int64_t T, int32_t K,
                          int32_t N, lbi_activation act, lbi_dtype dt, lbi_dtype out_dt,
                          void *workspace, size_t workspace_bytes, lbi_stream_t stream)
{
    if (!known(dt) || !known(out_dt) || !known_act(act))
        return LBI_ERR_DTYPE;
    if (bad_projection_shape(T, K, N))
        return LBI_ERR_SHAPE;
    if (T == 0)
        return LBI_OK;
    if (!x || !weight || !out)
        return LBI_ERR_NULL;
    ProductArgs a = forward_product(T, K, N, dt);
    const size_t need = (size_t)plan_product(a) * sizeof(float);
    lbi_status st = check_workspace(workspace, workspace_bytes, need);
    if (st != LBI_OK)
        return st;
    const size_t e = size_of(dt), oe = size_of(out_dt);
    const Tensor res = tokens(residual, T, N, ld_residual, oe), o = tokens(out, T, N, ld_out, oe);
    st = check_tensors({tokens(x, T, K, ld_x, e), tokens(weight, N, K, ld_weight, e),
                        dense(bias, 1, N, 4), res},
                       {o, tokens(pre, T, N, ld_pre, e),
                        dense(need ? workspace : nullptr, 1, (int64_t)need, 1)},
                       &o, &res);
    if (st != LBI_OK)
        return st;
    a.a = x; a.ld_a = ld_x;
    a.b = weight; a.ld_b = ld_weight;
    a.bias = bias;
    a.residual = residual; a.ld_residual = ld_residual;
    a.out = out; a.ld_out = ld_out;
    a.pre = pre; a.ld_pre = ld_pre;
    a.act = act;
    a.out_bf16 = out_dt == LBI_BF16;
    a.partial = (float *)workspace;
    return status_of(launch_product(a, (hipStream_t)stream));
}

size_t lbi_projection_backward_workspace_bytes(int64_t T, int32_t K, int32_t N,
                                               lbi_activation act, lbi_dtype dt,
                                               lbi_dtype out_dt)
{
    if (!known(dt) || !known(out_dt) || !known_act(act) || bad_projection_shape(T, K, N))
        return 0;
    return ProjectionGradient(T, K, N, act, dt, out_dt).layout(nullptr);
}

lbi_status lbi_projection_backward(const void *x, int64_t ld_x, const void *weight,
                                   int64_t ld_weight, const void *dout, int64_t ld_dout,
                                   const void *pre, int64_t ld_pre, void *dx, int64_t ld_dx,
                                   void *dweight, int64_t ld_dweight, float *dbias, int64_t T,
                                   int32_t K, int32_t N, lbi_activation act, lbi_dtype dt,
                                   lbi_dtype out_dt, void *workspace, size_t workspace_bytes,
                                   lbi_stream_t stream)
{
    if (!known(dt) || !known(out_dt) || !known_act(act))
        return LBI_ERR_DTYPE;
    if (bad_projection_shape(T, K, N))
        return LBI_ERR_SHAPE;
    if (act == LBI_ACT_NONE)
        pre = nullptr;
    if (T > 0 && (!dout || (act != LBI_ACT_NONE && !pre) || (dx && !weight) || (dweight && !x)))
        return LBI_ERR_NULL;
    ProjectionGradient p(T, K, N, act, dt, out_dt);
    const size_t need = p.layout(workspace), e = size_of(dt);
    lbi_status st = check_workspace(workspace, workspace_bytes, need);
    if (st != LBI_OK)
        return st;
    st = check_tensors({tokens(x, T, K, ld_x, e), tokens(weight, N, K, ld_weight, e),
                        tokens(dout, T, N, ld_dout, size_of(out_dt)), tokens(pre, T, N, ld_pre, e)},
                       {tokens(dx, T, K, ld_dx, e), tokens(dweight, N, K, ld_dweight, e),
                        dense(dbias, 1, N, 4),
                        dense(need ? workspace : nullptr, 1, (int64_t)need, 1)});
    if (st != LBI_OK)
        return st;
    const hipStream_t s = (hipStream_t)stream;
    p.slope.dout = dout; p.slope.ld_dout = ld_dout;
    p.slope.pre = pre; p.slope.ld_pre = ld_pre;
    const void *dz = dout;
    int64_t ld_dz = ld_dout;
    if (p.separate()) {
        dz = p.slope.dz;
        ld_dz = N;
    }
    if (!dbias)
        p.slope.partial = nullptr;
    hipError_t err = hipSuccess;
    if (p.separate() || dbias)
        err = launch_slope(p.slope, dbias, s);
    if (err == hipSuccess && dx && T > 0) {
        p.dx.a = dz; p.dx.ld_a = ld_dz;
        p.dx.b = weight; p.dx.ld_b = ld_weight;
        p.dx.out = dx; p.dx.ld_out = ld_dx;
        err = launch_product(p.dx, s);
    }
    if (err == hipSuccess && dweight) {
        if (T == 0)
            plan_product(p.dweight);
        p.dweight.a = dz; p.dweight.ld_a = ld_dz;
        p.dweight.b = x; p.dweight.ld_b = ld_x;
        p.dweight.out = dweight; p.dweight.ld_out = ld_dweight;
        err = launch_product(p.dweight, s);
    }
    return status_of(err);
}

size_t lbi_linear_attention_workspace_bytes(int64_t T, int64_t sequences, int32_t H, int32_t KH,
                                            int32_t DK, int32_t DV, int32_t ragged, lbi_dtype dt)
{
    if (!known(dt) || bad_attention_shape(T, sequences, H, KH, DK, DV, ragged != 0) ||
        sequences == 0)
        return 0;
    AttentionArgs a = {};
    a.in = attention_sizes(T, sequences, H, KH, DK, DV, dt);
    a.cut = attention_cut(a.in, ragged != 0, false);
    return attention_layout(a, nullptr);
}

lbi_status lbi_linear_attention(const lbi_attention_inputs *in, void *o, int64_t ld_o,
                                float *state_out, const int32_t *slots, int32_t n_slots,
                                void *workspace, size_t workspace_bytes, lbi_stream_t stream)
{
    lbi_status st = check_attention_inputs(in);
    if (st != LBI_OK)
        return st;
    if (slots && n_slots < 0)
        return LBI_ERR_SHAPE;
    if (in->sequences == 0)
        return LBI_OK;
    if (in->T > 0 && !o)
        return LBI_ERR_NULL;
    AttentionArgs a = {};
    a.in = *in;
    a.o = o; a.ld_o = ld_o;
    a.state_out = state_out;
    a.slots = slots; a.n_slots = n_slots;
    a.cut = attention_cut(*in, in->offsets != nullptr, false);
    const size_t need = attention_layout(a, workspace);
    if (!in->state_in || in->state_in != state_out)
        a.starts = nullptr;  // nothing writes what begins
    st = check_workspace(workspace, workspace_bytes, need);
    if (st != LBI_OK)
        return st;
    const int64_t rows = slots ? n_slots : in->sequences;
    const AttentionTensors t(*in, rows);
    const Tensor to = dense(state_out, rows, (int64_t)in->H * in->DK * in->DV, 4);
    st = check_tensors({t.q, t.k, t.v, t.decay, t.state, t.offsets,
                        dense(slots, 1, in->sequences, 4)},
                       {tokens(o, in->T, (int64_t)in->H * in->DV, ld_o, size_of(in->dt)), to,
                        dense(need ? workspace : nullptr, 1, (int64_t)need, 1)},
                       &to, &t.state);
    if (st != LBI_OK)
        return st;
    return status_of(launch_linear_attention(a, (hipStream_t)stream));
}

size_t lbi_linear_attention_backward_workspace_bytes(int64_t T, int64_t sequences, int32_t H,
                                                     int32_t KH, int32_t DK, int32_t DV,
                                                     int32_t ragged, lbi_dtype dt)
{
    if (!known(dt) || bad_attention_shape(T, sequences, H, KH, DK, DV, ragged != 0) ||
        sequences == 0)
        return 0;
    AttentionArgs a = {};
    a.in = attention_sizes(T, sequences, H, KH, DK, DV, dt);
    a.cut = attention_cut(a.in, ragged != 0, true);
    return attention_backward_layout(a, nullptr);
}

lbi_status lbi_linear_attention_backward(const lbi_attention_inputs *in, const void *dout,
                                         int64_t ld_dout, const float *dstate_out,
                                         const lbi_attention_gradients *grads, void *workspace,
                                         size_t workspace_bytes, lbi_stream_t stream)
{
    lbi_status st = check_attention_inputs(in);
    if (st != LBI_OK)
        return st;
    if (too_wide({ld_dout}))
        return LBI_ERR_SHAPE;
    if (!grads || (in->T > 0 && (!dout || !grads->dq || !grads->dk || !grads->dv)))
        return LBI_ERR_NULL;
    AttentionArgs a = {};
    a.in = *in;
    a.dout = dout; a.ld_dout = ld_dout;
    a.dstate_out = dstate_out;
    a.out = *grads;
    a.cut = attention_cut(*in, in->offsets != nullptr, true);
    const size_t need = attention_backward_layout(a, workspace);
    st = check_workspace(workspace, workspace_bytes, need);
    if (st != LBI_OK)
        return st;
    const AttentionTensors t(*in, in->sequences);
    const size_t e = size_of(in->dt);
    const int64_t T = in->T, hk = (int64_t)in->H * in->DK, hv = (int64_t)in->H * in->DV;
    const int64_t kk = (int64_t)in->KH * in->DK, kv = (int64_t)in->KH * in->DV;
    st = check_tensors({t.q, t.k, t.v, t.decay, t.state, t.offsets, tokens(dout, T, hv, ld_dout, e),
                        dense(dstate_out, in->sequences, hk * in->DV, 4)},
                       {tokens(a.out.dq, T, hk, a.out.ld_dq, e),
                        tokens(a.out.dk, T, kk, a.out.ld_dk, e),
                        tokens(a.out.dv, T, kv, a.out.ld_dv, e),
                        dense(a.out.dlog_decay, 1, in->H, 4),
                        dense(a.out.dstate_in, in->sequences, hk * in->DV, 4),
                        dense(need ? workspace : nullptr, 1, (int64_t)need, 1)});
    if (st != LBI_OK)
        return st;
    return status_of(launch_linear_attention_backward(a, (hipStream_t)stream));
}

lbi_status lbi_linear_attention_step(const lbi_attention_inputs *in, void *o, int64_t ld_o,
                                     float *state_out, const int32_t *slots, int32_t n_slots,
                                     lbi_stream_t stream)
{
    lbi_status st = check_attention_inputs(in);
    if (st != LBI_OK)
        return st;
    if (in->T != in->sequences || in->offsets || (slots && n_slots < 0))
        return LBI_ERR_SHAPE;
    if (in->sequences == 0)
        return LBI_OK;
    if (!o || !in->state_in || !state_out)
        return LBI_ERR_NULL;
    const int64_t rows = slots ? n_slots : in->sequences;
    const AttentionTensors t(*in, rows);
    const Tensor to = dense(state_out, rows, (int64_t)in->H * in->DK * in->DV, 4);
    st = check_tensors({t.q, t.k, t.v, t.decay, t.state, dense(slots, 1, in->sequences, 4)},
                       {tokens(o, in->T, (int64_t)in->H * in->DV, ld_o, size_of(in->dt)), to}, &to,
                       &t.state);
    if (st != LBI_OK)
        return st;
    AttentionArgs a = {};
    a.in = *in;
    a.o = o; a.ld_o = ld_o;
    a.state_out = state_out;
    a.slots = slots; a.n_slots = n_slots;
    return status_of(launch_linear_attention_step(a, (hipStream_t)stream));
}

}  // extern "C"
