// Gradient of linear attention.
//
// With S the state before a tile of n tokens, G the gradient of the state behind it and
// p_ij = scale a^(i-j) (q_i . k_j), e_ij = scale a^(i-j) (do_i . v_j) for j <= i:
//
//   dq_i = sum_{j <= i} e_ij k_j + scale a^(i+1) S do_i
//   dk_j = sum_{i >= j} e_ij q_i + a^(n-1-j) G v_j
//   dv_j = sum_{i >= j} p_ij do_i + a^(n-1-j) G^T k_j
//   G   <- a^n G + scale sum_i a^(i+1) q_i do_i^T
//   d log a = sum_ij (i-j) p_ij (do_i . v_j) + sum_i (i+1) scale a^(i+1) q_i S do_i
//             + sum_j (n-1-j) a^(n-1-j) k_j G v_j + n a^n <S, G>
//
// The last line differentiates every power of a where it stands, so that nothing in it cancels;
// it is formed from float32 sums of products of the inputs themselves.
//
// A workgroup takes a head along a range of tokens, twice: forwards for the states before its
// tiles, which it keeps in memory, then backwards with everything else.  G is held in both
// layouts, as the operand of G v and of G^T k.  States at the ranges' starts and gradients at
// their ends come from the kernels of the forward pass.
#include "lbi_attention.hpp"

namespace lbi {
namespace {

// Tokens of a tile: 64, or 32 where four float32 tiles of 128 values would not fit in LDS.
template <typename T, int DK, int DV>
constexpr int tile_tokens() { return sizeof(T) == 4 && DK + DV == 256 ? 32 : 64; }

template <typename T, int DK, int DV>
__global__ __launch_bounds__(256) void attention_backward_kernel(const AttentionArgs a,
                                                                 int64_t first, int marks)
{
    constexpr int C = tile_tokens<T, DK, DV>();
    constexpr int QS = tile_stride<T>(DK), VS = tile_stride<T>(DV), PS = tile_stride<T>(C);
    __shared__ __align__(16) T tile_q[C * QS], tile_k[C * QS], tile_v[C * VS], tile_d[C * VS];
    __shared__ __align__(16) T tile_p[C * PS], tile_e[C * PS];
    __shared__ int flags[4];
    __shared__ float sums[4];
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    const int h = blockIdx.x % a.in.H, kh = h / (a.in.H / a.in.KH);
    const int64_t range = first + blockIdx.x / a.in.H;
    const int dk = a.in.DK, dv = a.in.DV;
    const int64_t size = (int64_t)dk * dv;
    const float l2 = log2_decay(a.in.log_decay, h), scale = a.in.scale;
    const T *q0 = (const T *)a.in.q + h * dk, *k0 = (const T *)a.in.k + kh * dk;
    const T *v0 = (const T *)a.in.v + kh * dv, *d0 = (const T *)a.dout + h * dv;
    T *dq0 = (T *)a.out.dq + h * dk;
    const bool shared = a.part_k != nullptr;
    float *mark0 = a.marks + (range * a.in.H + h) * marks * size;

    const Sequences seqs = sequences_of(a.in);
    const Rows rows(a, range);
    Segment seg;
    auto state_in = [&](int64_t seq) {
        return a.in.state_in ? a.in.state_in + (seq * a.in.H + h) * size : nullptr;
    };
    // the state before the first tile of the segment that begins in the range at row `lo`
    auto begin = [&](int64_t lo) -> const float * {
        return seg.start < lo ? a.ends + ((range - 1) * a.in.H + h) * size : state_in(seg.seq);
    };
    State<T, DK, DV> state;
    float w[C / 4];

    // forwards: the states before the second and further tiles of each sequence
    seg.enter(seqs, rows.first, true);
    for (int64_t lo = rows.first; lo < rows.end;) {
        const int64_t hi = seg.end < rows.end ? seg.end : rows.end;
        if (hi - lo > C) {
            state.load(begin(lo), dk, dv, dv, 1);
            to_end<C>(w, l2, C);
            for (int64_t t = lo; t + C < hi; t += C) {
                load_tile<T, C, DK>(tile_k, k0 + t * a.in.ld_k, a.in.ld_k, C, dk);
                load_tile<T, C, DV>(tile_v, v0 + t * a.in.ld_v, a.in.ld_v, C, dv);
                __syncthreads();
                state.template update<C>(tile_k, tile_v, w, power(l2, (float)C));
                state.store(mark0 + ((t + C - rows.first) / C - 1) * size, dk, dv);
                __syncthreads();
            }
        }
        lo = hi;
        if (lo < rows.end)
            seg.advance(seqs);
    }
    __syncthreads();

    State<T, DK, DV> gb;  // G [dk][dv], a wavefront some columns dv
    State<T, DV, DK> ga;  // its transpose
    float decay = 0.f, decay_state = 0.f;

    // Tokens t .. t + n - 1 whose tiles are loaded, from the state at `before` ([dk][dv]).
    auto tile = [&](int64_t t, int n, const float *before) {
        causal_tiles<C>([&](int it, int jt) {
            f4 p = {0.f, 0.f, 0.f, 0.f}, e = {0.f, 0.f, 0.f, 0.f};
            if (jt <= it) {
#pragma unroll
                for (int b = 0; b < DK / 32; ++b) {
                    Frag<T> x, y;
                    x.rows(tile_k, QS, 16 * jt, 32 * b);
                    y.rows(tile_q, QS, 16 * it, 32 * b);
                    mma(p, x, y);
                }
#pragma unroll
                for (int b = 0; b < DV / 32; ++b) {
                    Frag<T> x, y;
                    x.rows(tile_v, VS, 16 * jt, 32 * b);
                    y.rows(tile_d, VS, 16 * it, 32 * b);
                    mma(e, x, y);
                }
                const int lag = 16 * (it - jt) + c16 - 4 * g;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float fade = power(l2, (float)(lag - r)) * scale;
                    p[r] = lag >= r ? p[r] * fade : 0.f;
                    decay += lag >= r ? (float)(lag - r) * p[r] * e[r] : 0.f;
                    e[r] = lag >= r ? e[r] * fade : 0.f;
                }
            }
            const int at = (16 * it + c16) * PS + 16 * jt + 4 * g;
            put4(tile_p + at, p);
            put4(tile_e + at, e);
        });
        __syncthreads();
        const float fade = power(l2, (float)n);
#pragma unroll
        for (int c = 0; c < DK / 64; ++c) {
            const int col = ga.column(c);
            {   // dq
                Wide<T, 2> fs[DV / 32];
#pragma unroll
                for (int b = 0; b < DV / 32; ++b) {
                    f4 x[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int at = 32 * b + 16 * u + 4 * g;
                        float y[4];
                        load_some<4>(before + (col + c16) * dv + at,
                                     before && col + c16 < dk ? dv - at : 0, y);
                        x[u] = f4{y[0], y[1], y[2], y[3]};
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            decay_state += (float)n * fade * y[r] * ga.s[2 * b + u][c][r];
                    }
                    pack_tiles(fs[b], x[0], x[1]);
                }
                Frag<T> fk[C / 32];
#pragma unroll
                for (int b = 0; b < C / 32; ++b)
                    fk[b].cols(tile_k, QS, 32 * b, col);
#pragma unroll 1
                for (int it = 0; it < C / 16; ++it) {
                    f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int b = 0; b < DV / 32; ++b) {
                        Frag<T> y;
                        y.rows(tile_d, VS, 16 * it, 32 * b);
                        mma(x, fs[b], y);
                    }
                    const int i = 16 * it + c16;
                    x *= power(l2, (float)(i + 1)) * scale;
                    const f4 q = get4(tile_q + i * QS + col + 4 * g);
                    decay += (float)(i + 1) * (x.x * q.x + x.y * q.y + x.z * q.z + x.w * q.w);
#pragma unroll
                    for (int b = 0; b < C / 32; ++b)
                        if (b <= it / 2) {
                            Frag<T> y;
                            y.rows(tile_e, PS, 16 * it, 32 * b);
                            mma(x, fk[b], y);
                        }
                    if (i < n)
                        store4(dq0 + (t + i) * a.out.ld_dq + col + 4 * g, dk - col - 4 * g, x);
                }
            }
            phase();
            {   // dk
                Wide<T, 2> fg[DV / 32];
#pragma unroll
                for (int b = 0; b < DV / 32; ++b)
                    pack_tiles(fg[b], ga.s[2 * b][c], ga.s[2 * b + 1][c]);
                Frag<T> fq[C / 32];
#pragma unroll
                for (int b = 0; b < C / 32; ++b)
                    fq[b].cols(tile_q, QS, 32 * b, col);
#pragma unroll 1
                for (int jt = 0; jt < C / 16; ++jt) {
                    f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int b = 0; b < DV / 32; ++b) {
                        Frag<T> y;
                        y.rows(tile_v, VS, 16 * jt, 32 * b);
                        mma(x, fg[b], y);
                    }
                    const int j = 16 * jt + c16;
                    const float left = (float)(n - 1 - j);
                    x *= j < n ? power(l2, left) : 0.f;
                    const f4 k = get4(tile_k + j * QS + col + 4 * g);
                    decay += j < n ? left * (x.x * k.x + x.y * k.y + x.z * k.z + x.w * k.w) : 0.f;
#pragma unroll
                    for (int b = 0; b < C / 32; ++b)
                        if (b >= jt / 2) {
                            Frag<T> y;
                            y.cols(tile_e, PS, 32 * b, 16 * jt);
                            mma(x, fq[b], y);
                        }
                    if (j >= n)
                        continue;
                    if (shared)
                        store4(a.part_k + ((t + j) * a.in.H + h) * dk + col + 4 * g,
                               dk - col - 4 * g, x);
                    else
                        store4((T *)a.out.dk + (t + j) * a.out.ld_dk + kh * dk + col + 4 * g,
                               dk - col - 4 * g, x);
                }
            }
        }
#pragma unroll
        for (int c = 0; c < DV / 64; ++c) {  // dv
            phase();
            const int col = gb.column(c);
            Wide<T, 2> fg[DK / 32];
#pragma unroll
            for (int b = 0; b < DK / 32; ++b)
                pack_tiles(fg[b], gb.s[2 * b][c], gb.s[2 * b + 1][c]);
            Frag<T> fd[C / 32];
#pragma unroll
            for (int b = 0; b < C / 32; ++b)
                fd[b].cols(tile_d, VS, 32 * b, col);
#pragma unroll 1
            for (int jt = 0; jt < C / 16; ++jt) {
                f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int b = 0; b < DK / 32; ++b) {
                    Frag<T> y;
                    y.rows(tile_k, QS, 16 * jt, 32 * b);
                    mma(x, fg[b], y);
                }
                const int j = 16 * jt + c16;
                x *= j < n ? power(l2, (float)(n - 1 - j)) : 0.f;
#pragma unroll
                for (int b = 0; b < C / 32; ++b)
                    if (b >= jt / 2) {
                        Frag<T> y;
                        y.cols(tile_p, PS, 32 * b, 16 * jt);
                        mma(x, fd[b], y);
                    }
                if (j >= n)
                    continue;
                if (shared)
                    store4(a.part_v + ((t + j) * a.in.H + h) * dv + col + 4 * g, dv - col - 4 * g,
                           x);
                else
                    store4((T *)a.out.dv + (t + j) * a.out.ld_dv + kh * dv + col + 4 * g,
                           dv - col - 4 * g, x);
            }
        }
        phase();
        from_start<C>(w, l2, n, scale);
        ga.template update<C>(tile_d, tile_q, w, fade);
        phase();
        gb.template update<C>(tile_q, tile_d, w, fade);
        __syncthreads();
    };
    auto load = [&](int64_t t, int n) {
        bool bad = load_tile<T, C, DK>(tile_q, q0 + t * a.in.ld_q, a.in.ld_q, n, dk);
        bad |= load_tile<T, C, DK>(tile_k, k0 + t * a.in.ld_k, a.in.ld_k, n, dk);
        bad |= load_tile<T, C, DV>(tile_v, v0 + t * a.in.ld_v, a.in.ld_v, n, dv);
        bad |= load_tile<T, C, DV>(tile_d, d0 + t * a.ld_dout, a.ld_dout, n, dv);
        return any_bad(bad, flags);
    };

    // backwards
    seg.enter(seqs, rows.end - 1, true);
    for (int64_t hi = rows.end; hi > rows.first;) {
        const int64_t lo = seg.start < rows.first ? rows.first : seg.start;
        const float *g0 = seg.end > rows.end
                              ? a.heads + ((range + 1) * a.in.H + h) * size
                              : (a.dstate_out ? a.dstate_out + (seg.seq * a.in.H + h) * size : nullptr);
        gb.load(g0, dk, dv, dv, 1);
        ga.load(g0, dv, dk, 1, dv);
        for (int64_t t = lo + (hi - lo - 1) / C * C; t >= lo; t -= C) {
            const int n = hi - t < C ? (int)(hi - t) : C;
            const float *before =
                t > lo ? mark0 + ((t - rows.first) / C - 1) * size : begin(lo);
            // Where a value is infinite or NaN: token by token, each from the state that the ones
            // before it in the tile leave, which 0 times it must not reach.
            const bool bad = load(t, n);
            float *scratch = mark0 + (int64_t)(marks - 1) * size;
            for (int i = bad ? n - 1 : 0; i >= 0; --i) {
                const float *from = before;
                if (bad) {
                    __syncthreads();
                    if (i > 0) {
                        load(t, i);
                        state.load(before, dk, dv, dv, 1);
                        to_end<C>(w, l2, i);
                        state.template update<C>(tile_k, tile_v, w, power(l2, (float)i));
                        state.store(scratch, dk, dv);
                        from = scratch;
                        __syncthreads();
                    }
                    load(t + i, 1);
                }
                tile(t + i, bad ? 1 : n, from);
            }
        }
        if (lo == seg.start && a.out.dstate_in)
            gb.store(a.out.dstate_in + (seg.seq * a.in.H + h) * size, dk, dv);
        hi = lo;
        if (hi > rows.first)
            seg.enter(seqs, hi - 1, true);
    }
    if (!a.part_decay)
        return;
    decay = lanes_sum<64>(decay + decay_state);
    if (lane == 0)
        sums[threadIdx.x >> 6] = decay;
    __syncthreads();
    if (threadIdx.x == 0)
        a.part_decay[range * a.in.H + h] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// The gradients of shared keys and values: the sums over the heads that share them.
template <typename T>
__global__ __launch_bounds__(256) void shared_heads_kernel(const float *part, T *out, int64_t ld,
                                                           int64_t T0, int64_t count, int KH,
                                                           int share, int width)
{
    const int64_t per = (int64_t)KH * width;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < count * per;
         id += (int64_t)gridDim.x * 256) {
        const int64_t t = T0 + id / per;
        const int at = (int)(id % per), kh = at / width, d = at % width;
        const float *p = part + (t * KH + kh) * share * width + d;
        float v = p[0];
        for (int s = 1; s < share; ++s)
            v += p[s * width];
        out[t * ld + at] = narrow<T>(v);
    }
}

struct ToVector {
    float *out;
    __device__ __forceinline__ void operator()(int64_t c, float v) const { out[c] = v; }
};

}  // namespace

int64_t attention_marks(const lbi_attention_inputs &in, const AttentionCut &cut)
{
    int64_t marks = 0;
    (void)by_head(in, [&](auto type, auto dk, auto dv) {
        marks = cut.tokens /
                tile_tokens<decltype(type), decltype(dk)::value, decltype(dv)::value>();
        return hipSuccess;
    });
    return marks;
}

hipError_t launch_linear_attention_backward(const AttentionArgs &a, hipStream_t stream)
{
    hipError_t e = hipSuccess;
    if (a.in.T > 0) {
        if (a.cut.joined) {
            e = launch_attention_ends(a, false, stream);
            if (e == hipSuccess)
                e = launch_attention_ends(a, true, stream);
        }
        if (e == hipSuccess)
            e = by_head(a.in, [&](auto type, auto dk, auto dv) {
                using T = decltype(type);
                constexpr int DK = decltype(dk)::value, DV = decltype(dv)::value;
                const int marks = (int)attention_marks(a.in, a.cut);
                return in_launches(a.cut.ranges, a.in.H, [&](int64_t first, dim3 grid) {
                    attention_backward_kernel<T, DK, DV><<<grid, 256, 0, stream>>>(a, first, marks);
                });
            });
        if (e != hipSuccess)
            return e;
        if (a.part_k) {
            const int share = a.in.H / a.in.KH;
            auto sum = [&](auto type, const float *part, void *out, int64_t ld, int width) {
                using T = decltype(type);
                const int64_t n = (a.in.T * a.in.KH * width + 255) / 256;
                shared_heads_kernel<T><<<dim3((unsigned)(n < 8192 ? n : 8192)), 256, 0, stream>>>(
                    part, (T *)out, ld, 0, a.in.T, a.in.KH, share, width);
            };
            if (a.in.dt == LBI_BF16) {
                sum(bf16_bits{}, a.part_k, a.out.dk, a.out.ld_dk, a.in.DK);
                sum(bf16_bits{}, a.part_v, a.out.dv, a.out.ld_dv, a.in.DV);
            } else {
                sum(float{}, a.part_k, a.out.dk, a.out.ld_dk, a.in.DK);
                sum(float{}, a.part_v, a.out.dv, a.out.ld_dv, a.in.DV);
            }
            e = hipGetLastError();
        }
    }
    if (e == hipSuccess && a.out.dlog_decay)
        e = sum_rows(a.part_decay, a.in.T > 0 ? a.cut.ranges : 0, a.in.H, a.in.H,
                     ToVector{a.out.dlog_decay}, stream);
    if (e == hipSuccess && a.out.dstate_in && (a.in.offsets || a.in.T == 0))
        e = launch_attention_empty(a, true, stream);
    return e;
}

}  // namespace lbi
