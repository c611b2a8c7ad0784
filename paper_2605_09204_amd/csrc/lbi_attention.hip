// Linear attention with a decay for each head: forward over packed sequences, and single tokens.
//
//   S_t = a S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t
//
// A workgroup takes a head along a range of tokens, in tiles of n <= 64 that hold one sequence's.
// With S the state before a tile and i, j its tokens from 0,
//
//   o_i = scale (a^(i+1) q_i^T S + sum_{j <= i} a^(i-j) (q_i . k_j) v_j),
//   S  <- a^n S + sum_j a^(n-1-j) k_j v_j^T:
//
// four matrix products a tile, all powers of a at most 1.  The state stays in registers, where its
// layout is that of an operand.  Where sequences and heads are too few to fill the GPU, ranges
// are shorter than sequences: a first kernel forms the state that each range adds, a second one
// carries states along the ranges, and the third walks again from there with outputs.
//
// A value that is infinite or NaN would reach earlier tokens of its tile (0 times it is NaN), so
// tiles with one are taken token by token.
#include "lbi_attention.hpp"

namespace lbi {
namespace {

constexpr int C = kAttentionTile;

template <typename T, int DK, int DV>
__global__ __launch_bounds__(256, (sizeof(T) == 2 || DK + DV == 128) ? 2 : 1) void attention_kernel(const AttentionArgs a, int64_t first)
{
    constexpr int QS = tile_stride<T>(DK), VS = tile_stride<T>(DV), PS = tile_stride<T>(C);
    __shared__ __align__(16) T tile_q[C * QS], tile_k[C * QS], tile_v[C * VS], tile_p[C * PS];
    __shared__ int flags[4];
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    const int h = blockIdx.x % a.in.H, kh = h / (a.in.H / a.in.KH);
    const int64_t range = first + blockIdx.x / a.in.H;
    const int dk = a.in.DK, dv = a.in.DV;
    const int64_t size = (int64_t)dk * dv;
    const float l2 = log2_decay(a.in.log_decay, h), scale = a.in.scale;
    const T *q0 = (const T *)a.in.q + h * dk, *k0 = (const T *)a.in.k + kh * dk;
    const T *v0 = (const T *)a.in.v + kh * dv;
    T *o0 = (T *)a.o + h * dv;

    const Sequences seqs = sequences_of(a.in);
    const Rows rows(a, range);
    Segment seg;
    seg.enter(seqs, rows.first, true);
    State<T, DK, DV> state;
    auto begin = [&] {
        const int64_t row = a.in.state_in ? state_row(a.slots, a.n_slots, seg.seq) : -1;
        const float *p = row >= 0 ? a.in.state_in + (row * a.in.H + h) * size : nullptr;
        if (a.starts && seg.end > rows.end)  // another workgroup may have written the slot
            p = a.starts + (range * a.in.H + h) * size;
        state.load(p, dk, dv, dv, 1);
    };
    if (seg.start < rows.first)
        state.load(a.ends + ((range - 1) * a.in.H + h) * size, dk, dv, dv, 1);
    else
        begin();
    float w[C / 4];
    int weights_of = 0;
    for (int64_t t = rows.first; t < rows.end;) {
        const int64_t stop = seg.end < rows.end ? seg.end : rows.end;
        int n = stop - t < C ? (int)(stop - t) : C;
        auto load = [&](int n) {
            bool bad = load_tile<T, C, DK>(tile_q, q0 + t * a.in.ld_q, a.in.ld_q, n, dk);
            bad |= load_tile<T, C, DK>(tile_k, k0 + t * a.in.ld_k, a.in.ld_k, n, dk);
            bad |= load_tile<T, C, DV>(tile_v, v0 + t * a.in.ld_v, a.in.ld_v, n, dv);
            return any_bad(bad, flags);
        };
        if (load(n) && n > 1) {
            n = 1;
            __syncthreads();
            load(n);
        }
        if (n != weights_of) {
            to_end<C>(w, l2, n);
            weights_of = n;
        }
        // p_ij = scale a^(i-j) q_i . k_j, rounded to the tokens' type as an operand
        causal_tiles<C>([&](int it, int jt) {
            f4 p = {0.f, 0.f, 0.f, 0.f};
            if (jt <= it) {
#pragma unroll
                for (int b = 0; b < DK / 32; ++b) {
                    Frag<T> fq, fk;
                    fk.rows(tile_k, QS, 16 * jt, 32 * b);
                    fq.rows(tile_q, QS, 16 * it, 32 * b);
                    mma(p, fk, fq);
                }
                const int lag = 16 * (it - jt) + c16 - 4 * g;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    p[r] = lag >= r ? p[r] * (power(l2, (float)(lag - r)) * scale) : 0.f;
            }
            put4(tile_p + (16 * it + c16) * PS + 16 * jt + 4 * g, p);
        });
        __syncthreads();
#pragma unroll
        for (int c = 0; c < DV / 64; ++c) {
            const int col = state.column(c);
            Frag<T> fv[C / 32];
#pragma unroll
            for (int b = 0; b < C / 32; ++b)
                fv[b].cols(tile_v, VS, 32 * b, col);
            Wide<T, 2> fs[DK / 32];
#pragma unroll
            for (int b = 0; b < DK / 32; ++b)
                pack_tiles(fs[b], state.s[2 * b][c], state.s[2 * b + 1][c]);
#pragma unroll 1
            for (int it = 0; it < C / 16; ++it) {
                f4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int b = 0; b < DK / 32; ++b) {
                    Frag<T> fq;
                    fq.rows(tile_q, QS, 16 * it, 32 * b);
                    mma(o, fs[b], fq);
                }
                const int i = 16 * it + c16;
                o *= power(l2, (float)(i + 1)) * scale;
#pragma unroll
                for (int b = 0; b < C / 32; ++b)
                    if (b <= it / 2) {
                        Frag<T> fp;
                        fp.rows(tile_p, PS, 16 * it, 32 * b);
                        mma(o, fv[b], fp);
                    }
                if (i < n)
                    store4(o0 + (t + i) * a.ld_o + col + 4 * g, dv - col - 4 * g, o);
            }
        }
        phase();
        state.template update<C>(tile_k, tile_v, w, power(l2, (float)n));
        t += n;
        if (t == seg.end) {
            if (a.state_out) {
                const int64_t row = state_row(a.slots, a.n_slots, seg.seq);
                if (row >= 0)
                    state.store(a.state_out + (row * a.in.H + h) * size, dk, dv);
            }
            if (t < rows.end) {
                seg.advance(seqs);
                begin();
            }
        }
        __syncthreads();
    }
}

// What a range adds to the state of the sequence that passes its end (states), or to the gradient
// of the state of the sequence that passes its start.
template <typename T, int DK, int DV>
__global__ __launch_bounds__(256) void ends_kernel(const AttentionArgs a, int64_t first,
                                                   bool backward)
{
    constexpr int QS = tile_stride<T>(DK), VS = tile_stride<T>(DV);
    __shared__ __align__(16) T tile_a[C * QS], tile_b[C * VS];
    const int h = blockIdx.x % a.in.H, kh = h / (a.in.H / a.in.KH);
    const int64_t range = first + blockIdx.x / a.in.H;
    const int dk = a.in.DK, dv = a.in.DV;
    const int64_t size = (int64_t)dk * dv;
    const float l2 = log2_decay(a.in.log_decay, h);
    const Sequences seqs = sequences_of(a.in);
    const Rows rows(a, range);
    Segment seg;
    seg.enter(seqs, backward ? rows.first : rows.end - 1, true);
    const bool before = seg.start < rows.first, behind = seg.end > rows.end;
    int32_t *flag = (backward ? a.head_flags : a.end_flags) + range;
    if (backward ? !before : !behind) {
        if (h == 0 && threadIdx.x == 0)
            *flag = 0;
        return;
    }
    if (h == 0 && threadIdx.x == 0)
        *flag = before && behind ? kWhole : kPart;
    const int64_t from = before ? rows.first : seg.start, to = behind ? rows.end : seg.end;
    State<T, DK, DV> state;
    float w[C / 4];
    if (!backward) {
        const int64_t row = !before && a.in.state_in ? state_row(a.slots, a.n_slots, seg.seq) : -1;
        state.load(row >= 0 ? a.in.state_in + (row * a.in.H + h) * size : nullptr, dk, dv, dv, 1);
        if (a.starts && !before)
            state.store(a.starts + (range * a.in.H + h) * size, dk, dv);
        const T *k0 = (const T *)a.in.k + kh * dk, *v0 = (const T *)a.in.v + kh * dv;
        for (int64_t t = from; t < to; t += C) {
            const int n = to - t < C ? (int)(to - t) : C;
            load_tile<T, C, DK>(tile_a, k0 + t * a.in.ld_k, a.in.ld_k, n, dk);
            load_tile<T, C, DV>(tile_b, v0 + t * a.in.ld_v, a.in.ld_v, n, dv);
            if (t == from || n < C)
                to_end<C>(w, l2, n);
            __syncthreads();
            state.template update<C>(tile_a, tile_b, w, power(l2, (float)n));
            __syncthreads();
        }
    } else {
        state.load(!behind && a.dstate_out ? a.dstate_out + (seg.seq * a.in.H + h) * size : nullptr,
                   dk, dv, dv, 1);
        const T *q0 = (const T *)a.in.q + h * dk, *d0 = (const T *)a.dout + h * dv;
        for (int64_t t = from + (to - from - 1) / C * C; t >= from; t -= C) {
            const int n = to - t < C ? (int)(to - t) : C;
            load_tile<T, C, DK>(tile_a, q0 + t * a.in.ld_q, a.in.ld_q, n, dk);
            load_tile<T, C, DV>(tile_b, d0 + t * a.ld_dout, a.ld_dout, n, dv);
            from_start<C>(w, l2, n, a.in.scale);
            __syncthreads();
            state.template update<C>(tile_a, tile_b, w, power(l2, (float)n));
            __syncthreads();
        }
    }
    state.store((backward ? a.heads : a.ends) + (range * a.in.H + h) * size, dk, dv);
}

// States along the ranges of a sequence (of all tokens, with offsets), or their gradients against
// them: one thread for each value of each head.
__global__ __launch_bounds__(256) void carry_kernel(const AttentionArgs a, int64_t first,
                                                    int blocks, bool backward)
{
    const int64_t size = (int64_t)a.in.DK * a.in.DV;
    const uint32_t id = blockIdx.x;
    const int64_t e = (int64_t)(id % blocks) * 256 + threadIdx.x;
    const int h = id / blocks % a.in.H;
    const int64_t chain = first + id / blocks / a.in.H;
    if (e >= size)
        return;
    const int64_t count = a.cut.per_sequence > 0 ? a.cut.per_sequence : a.cut.ranges;
    const float fade = power(log2_decay(a.in.log_decay, h), (float)a.cut.tokens);
    float *p = (backward ? a.heads : a.ends) + h * size + e;
    const int32_t *flags = backward ? a.head_flags : a.end_flags;
    const int64_t step = a.in.H * size;
    float v = 0.f;
    constexpr int AHEAD = 8;
    for (int64_t i = 0; i < count; i += AHEAD) {
        float x[AHEAD];
        int32_t f[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int64_t r = chain * count + (backward ? count - 1 - i - k : i + k);
            const bool there = i + k < count;
            f[k] = there ? flags[r] : 0;
            x[k] = f[k] ? p[r * step] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int64_t r = chain * count + (backward ? count - 1 - i - k : i + k);
            v = f[k] == kWhole ? x[k] + fade * v : x[k];
            if (f[k] == kWhole)
                p[r * step] = v;
        }
    }
}

__global__ __launch_bounds__(256) void empty_kernel(const AttentionArgs a, int64_t first,
                                                    bool backward)
{
    const int64_t seq = first + blockIdx.x / a.in.H;
    const int h = blockIdx.x % a.in.H;
    const Sequences seqs = sequences_of(a.in);
    if (seqs.at(seq + 1) > seqs.at(seq))
        return;
    const int64_t size = (int64_t)a.in.DK * a.in.DV;
    const int64_t row = backward ? seq : state_row(a.slots, a.n_slots, seq);
    if (row < 0)
        return;
    const float *from = backward ? a.dstate_out : a.in.state_in;
    float *to = (backward ? a.out.dstate_in : a.state_out) + (row * a.in.H + h) * size;
    for (int64_t e = threadIdx.x; e < size; e += 256)
        to[e] = from ? from[(row * a.in.H + h) * size + e] : 0.f;
}

// One token: a workgroup takes a head of a sequence, COLS lanes of 4 columns side by side, the
// other lanes further rows.  Bound by the state, which is read and written once.
template <typename T, int COLS>
__global__ __launch_bounds__(256) void step_kernel(const AttentionArgs a, int64_t first)
{
    constexpr int ROWS = 256 / COLS;
    __shared__ float sums[ROWS][COLS * 4 + 1];
    const int h = blockIdx.x % a.in.H, kh = h / (a.in.H / a.in.KH);
    const int64_t seq = first + blockIdx.x / a.in.H;
    const int dk = a.in.DK, dv = a.in.DV;
    const int64_t size = (int64_t)dk * dv;
    const int col = threadIdx.x % COLS * 4, row0 = threadIdx.x / COLS;
    const float fade = power(log2_decay(a.in.log_decay, h), 1.f);
    const T *q = (const T *)a.in.q + seq * a.in.ld_q + h * dk;
    const T *k = (const T *)a.in.k + seq * a.in.ld_k + kh * dk;
    float v[4], o[4] = {0.f, 0.f, 0.f, 0.f};
    load_some<4>((const T *)a.in.v + seq * a.in.ld_v + kh * dv + col, dv - col, v);
    const int64_t slot = state_row(a.slots, a.n_slots, seq);
    const float *from = a.in.state_in + (slot * a.in.H + h) * size;
    float *to = a.state_out + (slot * a.in.H + h) * size;
    constexpr int DEEP = 8;
    for (int i0 = row0; i0 < dk; i0 += DEEP * ROWS) {
        float s[DEEP][4], kk[DEEP], qq[DEEP];
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            const int i = i0 + d * ROWS;
            load_some<4>(from + i * dv + col, slot >= 0 && i < dk ? dv - col : 0, s[d]);
            kk[d] = i < dk ? widen(k[i]) : 0.f;
            qq[d] = i < dk ? widen(q[i]) : 0.f;
        }
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            const int i = i0 + d * ROWS;
            if (i >= dk)
                break;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                s[d][c] = fade * s[d][c] + kk[d] * v[c];
                o[c] += qq[d] * s[d][c];
            }
            if (slot >= 0)
                store_some<4>(to + i * dv + col, dv - col, s[d]);
        }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
        sums[row0][col + c] = o[c];
    __syncthreads();
    if ((int)threadIdx.x < dv) {
        float s = 0.f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            s += sums[r][threadIdx.x];
        ((T *)a.o)[seq * a.ld_o + h * dv + threadIdx.x] = narrow<T>(s * a.in.scale);
    }
}

}  // namespace

AttentionCut attention_cut(const lbi_attention_inputs &in, bool ragged)
{
    AttentionCut c = {};
    if (in.T == 0)
        return c;
    // about three workgroups a CU
    const int64_t want = (768 + in.H - 1) / in.H;
    if (!ragged) {
        const int64_t len = in.T / in.sequences;
        int64_t per = in.sequences >= want ? 1 : (want + in.sequences - 1) / in.sequences;
        c.tokens = ((len + per - 1) / per + kAttentionTile - 1) / kAttentionTile * kAttentionTile;
        per = (len + c.tokens - 1) / c.tokens;
        c.per_sequence = (int32_t)per;
        c.ranges = in.sequences * per;
        c.joined = per > 1;
    } else {
        c.tokens = ((in.T + want - 1) / want + kAttentionTile - 1) / kAttentionTile * kAttentionTile;
        c.ranges = (in.T + c.tokens - 1) / c.tokens;
        c.joined = c.ranges > 1;
    }
    return c;
}

hipError_t launch_attention_ends(const AttentionArgs &a, bool backward, hipStream_t stream)
{
    hipError_t e = by_head(a.in, [&](auto type, auto dk, auto dv) {
        return in_launches(a.cut.ranges, a.in.H, [&](int64_t first, dim3 grid) {
            ends_kernel<decltype(type), decltype(dk)::value, decltype(dv)::value>
                <<<grid, 256, 0, stream>>>(a, first, backward);
        });
    });
    if (e != hipSuccess)
        return e;
    const int64_t size = (int64_t)a.in.DK * a.in.DV;
    const int blocks = (int)((size + 255) / 256);
    const int64_t chains = a.cut.per_sequence > 0 ? a.in.sequences : 1;
    return in_launches(chains, (int64_t)blocks * a.in.H, [&](int64_t first, dim3 grid) {
        carry_kernel<<<grid, 256, 0, stream>>>(a, first, blocks, backward);
    });
}

hipError_t launch_attention_empty(const AttentionArgs &a, bool backward, hipStream_t stream)
{
    return in_launches(a.in.sequences, a.in.H, [&](int64_t first, dim3 grid) {
        empty_kernel<<<grid, 256, 0, stream>>>(a, first, backward);
    });
}

hipError_t launch_linear_attention(const AttentionArgs &a, hipStream_t stream)
{
    hipError_t e = hipSuccess;
    if (a.in.T > 0) {
        if (a.cut.joined)
            e = launch_attention_ends(a, false, stream);
        if (e == hipSuccess)
            e = by_head(a.in, [&](auto type, auto dk, auto dv) {
                return in_launches(a.cut.ranges, a.in.H, [&](int64_t first, dim3 grid) {
                    attention_kernel<decltype(type), decltype(dk)::value, decltype(dv)::value>
                        <<<grid, 256, 0, stream>>>(a, first);
                });
            });
        if (e != hipSuccess)
            return e;
    }
    if (a.state_out && a.state_out != a.in.state_in && (a.in.offsets || a.in.T == 0))
        e = launch_attention_empty(a, false, stream);
    return e;
}

hipError_t launch_linear_attention_step(const AttentionArgs &a, hipStream_t stream)
{
    return in_launches(a.in.sequences, a.in.H, [&](int64_t first, dim3 grid) {
        const bool narrow_rows = a.in.DV <= 64;
        if (a.in.dt == LBI_BF16) {
            if (narrow_rows) step_kernel<bf16_bits, 16><<<grid, 256, 0, stream>>>(a, first);
            else step_kernel<bf16_bits, 32><<<grid, 256, 0, stream>>>(a, first);
        } else {
            if (narrow_rows) step_kernel<float, 16><<<grid, 256, 0, stream>>>(a, first);
            else step_kernel<float, 32><<<grid, 256, 0, stream>>>(a, first);
        }
    });
}

}  // namespace lbi
