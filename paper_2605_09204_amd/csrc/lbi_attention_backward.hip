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
// A first kernel walks forwards along each range of tokens and leaves the states before its tiles
// in memory; then a workgroup takes a head along a range backwards with everything else.  G is
// held in both layouts, as the operand of G v and of G^T k.  The states that enter the ranges and
// the gradients that leave them are carried as in the forward pass.
//
// 8 sequences of 2048 tokens, 12 heads of 64, bf16: 96 to 99 us for the walk (226 MB with the kept
// states), 37 for both sides of the ranges, 6 for the carry.  The walk's wavefronts wait 44 per cent
// of their cycles, on LDS (39 per cent of its cycles are bank conflicts) and on products in a chain, at
// the two workgroups a CU that the registers leave, and issue 11 vector instructions for each of the
// matrix cores'.
#include "lbi_attention.hpp"

namespace lbi {
namespace {

// Tokens of a tile: 64, or 32 of float32, of which LDS and the registers hold two workgroups a CU
// (heads of 256 values together: one), not one.  3885 tokens, 6 heads of 48 and 101: 131 us -> 88.
template <typename T, int DK, int DV>
constexpr int tile_tokens() { return sizeof(T) == 4 ? 32 : 64; }

template <typename T, int DK, int DV, bool FULL>
__global__ __launch_bounds__(256, DK + DV <= (sizeof(T) == 2 ? 128 : 192) ? 2 : 1) void
attention_backward_kernel(const AttentionArgs a, int64_t first, int marks)
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
    const int dk = FULL ? DK : a.in.DK, dv = FULL ? DV : a.in.DV;
    const int64_t size = (int64_t)dk * dv;
    const float l2 = log2_decay(a.in.log_decay, h), scale = a.in.scale;
    const T *q0 = (const T *)a.in.q + h * dk, *k0 = (const T *)a.in.k + kh * dk;
    const T *v0 = (const T *)a.in.v + kh * dv, *d0 = (const T *)a.dout + h * dv;
    T *dq0 = (T *)a.out.dq + h * dk;
    const bool shared = a.part_k != nullptr;
    float *mark0 = a.marks + (range * a.in.H + h) * marks * size;

    const Sequences seqs = sequences_of(a.in);
    const Rows rows(a, range);
    float w[C / 4];
    State<T, DK, DV, FULL> gb;  // G [dk][dv], a wavefront some columns dv
    State<T, DV, DK, FULL> ga;  // its transpose
    float decay = 0.f, decay_state = 0.f;
    f4 causal[kCausalTiles<C>];
    causal_fade<C>(causal, l2, scale);

    // The state before a tile: what its range or its sequence's first state adds, and what enters
    // the range; either may be NULL.
    struct Before {
        const float *own, *entering;
        float fade;  // of what enters
    };

    // This wavefront's part of that state as the operand of S do, from column c on.
    auto fetch = [&](const Before &b, int c, float (&x)[DV / 16][4], float (&y)[DV / 16][4]) {
        const int row = ga.column(c) + c16;
#pragma unroll
        for (int u = 0; u < DV / 16; ++u) {
            const int at = 16 * u + 4 * g, left = FULL ? 4 : row < dk ? dv - at : 0;
            load_some<4>(b.own + row * dv + at, b.own ? left : 0, x[u]);
            load_some<4>(b.entering + row * dv + at, b.entering ? left : 0, y[u]);
        }
    };

    // With keys or values of 128 the registers do not hold what is on its way as well.
    constexpr bool AHEAD = FULL && DK + DV == 128;

    // Tokens t .. t + n - 1 whose tiles are loaded; halfway() is called when dq and dk are done.  States
    // go into dq and dk as three bf16 values, since d log a takes its part of them from there: with two
    // it was off by up to 5e-6, several times what sums of float32 products are.
    auto tile = [&](int64_t t, int n, const Before &before, auto &&halfway) {
        float own[DV / 16][4], entering[DV / 16][4];
        if (AHEAD)
            fetch(before, 0, own, entering);
        causal_tiles<C>([&](int at, int it, int jt) {
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
                    p[r] = lag >= r ? p[r] * causal[at][r] : 0.f;
                    decay += lag >= r ? (float)(lag - r) * p[r] * e[r] : 0.f;
                    e[r] = lag >= r ? e[r] * causal[at][r] : 0.f;
                }
            }
            // operands, rounded to the tokens' type (bf16: the gradients' error against float64 is
            // 0.0018, of which their own rounding is 0.0017; the decay's took p and e as they were)
            const int to = (16 * it + c16) * PS + 16 * jt + lane_quad<T>();
            put4(tile_p + to, p);
            put4(tile_e + to, e);
        });
        __syncthreads();
        const float fade = power(l2, (float)n);
#pragma unroll
        for (int c = 0; c < DK / 64; ++c) {
            const int col = ga.column(c);
            {   // dq
                if (!AHEAD)
                    fetch(before, c, own, entering);
                Wide<T, 3> fs[DV / 32];
                float inner = 0.f;
#pragma unroll
                for (int b = 0; b < DV / 32; ++b) {
                    f4 x[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            x[u][r] = own[2 * b + u][r] + before.fade * entering[2 * b + u][r];
                            inner += x[u][r] * ga.s[2 * b + u][c][r];
                        }
                    pack_tiles(fs[b], x[0], x[1]);
                }
                decay_state += (float)n * fade * inner;
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
                    const f4 q = get4(tile_q + i * QS + col + lane_quad<T>());
                    decay += (float)(i + 1) * (x.x * q.x + x.y * q.y + x.z * q.z + x.w * q.w);
#pragma unroll
                    for (int b = 0; b < C / 32; ++b)
                        if (b <= it / 2) {
                            Frag<T> y;
                            y.rows(tile_e, PS, 16 * it, 32 * b);
                            mma(x, fk[b], y);
                        }
                    if (i < n)
                        store4<T, FULL>(dq0 + (t + i) * a.out.ld_dq + col + 4 * g, dk - col - 4 * g, x);
                }
            }
            phase();
            {   // dk
                Wide<T, 3> fg[DV / 32];
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
                    const f4 k = get4(tile_k + j * QS + col + lane_quad<T>());
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
                        store4<float, FULL>(a.part_k + ((t + j) * a.in.H + h) * dk + col + 4 * g,
                               dk - col - 4 * g, x);
                    else
                        store4<T, FULL>((T *)a.out.dk + (t + j) * a.out.ld_dk + kh * dk + col + 4 * g,
                               dk - col - 4 * g, x);
                }
            }
        }
        halfway();
#pragma unroll
        for (int c = 0; c < DV / 64; ++c) {  // dv
            phase();
            const int col = gb.column(c);
            Wide<T, 2> fg[DK / 32];  // two: dv is rounded to 2^-8 behind it, and goes nowhere else
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
                    store4<float, FULL>(a.part_v + ((t + j) * a.in.H + h) * dv + col + 4 * g, dv - col - 4 * g,
                           x);
                else
                    store4<T, FULL>((T *)a.out.dv + (t + j) * a.out.ld_dv + kh * dv + col + 4 * g,
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
    TileLoad<T, C, DK, FULL> next_q, next_k;
    TileLoad<T, C, DV, FULL> next_v, next_d;
    auto load = [&](int64_t t, int n) {
        next_q.load(q0 + t * a.in.ld_q, a.in.ld_q, n, dk);
        next_k.load(k0 + t * a.in.ld_k, a.in.ld_k, n, dk);
        next_v.load(v0 + t * a.in.ld_v, a.in.ld_v, n, dv);
        next_d.load(d0 + t * a.ld_dout, a.ld_dout, n, dv);
    };
    auto put = [&] {
        bool bad = next_q.put(tile_q);
        bad |= next_k.put(tile_k);
        bad |= next_v.put(tile_v);
        bad |= next_d.put(tile_d);
        return any_bad(bad, flags);
    };
    // The tiles from the range's end to its start: rows t .. t + n - 1 of seg, which has the rows
    // from lo on in the range.
    Segment seg;
    int64_t lo = rows.end, t = rows.end;
    enum Kind { kNone, kTile, kState };
    struct Item {
        Kind kind;
        int64_t t, seq;
        int n;
        bool fresh, begins, behind;  // its sequence's last rows, its first ones; it leaves the range
        Before before;
    };
    auto step = [&]() -> Item {
        if (t <= rows.first)
            return {};
        Item x;
        x.kind = kTile;
        x.fresh = t == lo;
        if (t > lo) {
            t -= C;
            x.n = C;
        } else {
            const int64_t hi = lo;
            seg.enter(seqs, hi - 1, true);
            lo = seg.start < rows.first ? rows.first : seg.start;
            t = lo + (hi - lo - 1) / C * C;
            x.n = (int)(hi - t);
        }
        x.t = t;
        x.seq = seg.seq;
        x.begins = t == lo && lo == seg.start;
        x.behind = seg.end > rows.end;
        x.before = {nullptr, nullptr, power(l2, (float)(t - lo))};
        if (t > lo)
            x.before.own = mark0 + ((t - rows.first) / C - 1) * size;
        else if (lo == seg.start && a.in.state_in)
            x.before.own = a.in.state_in + (seg.seq * a.in.H + h) * size;
        if (seg.start < lo)
            x.before.entering = a.ends + ((range - 1) * a.in.H + h) * size;
        return x;
    };
    // A tile with a value that is infinite or NaN is taken token by token, the last one first, each
    // from the state that the ones before it in the tile leave, which 0 times it must not reach: for
    // that state their rows are loaded once (kState), then the token itself.
    float *scratch = mark0 + (int64_t)(marks - 1) * size;
    Item now = {}, next = step(), whole = {};
    int single = -1;  // the token of `whole` that is next
    while (true) {
        if (now.kind == kTile) {
            if (now.fresh) {
                const float *p = now.behind       ? a.heads + ((range + 1) * a.in.H + h) * size
                                 : a.dstate_out ? a.dstate_out + (now.seq * a.in.H + h) * size
                                                : nullptr;
                gb.load(p, dk, dv, dv, 1);
                ga.load(p, dv, dk, 1, dv);
            }
            tile(now.t, now.n, now.before, [&] {
                if (AHEAD)  // on its way for the rest of the tile in LDS (none: its rows again, unused)
                    load(next.kind == kNone ? now.t : next.t, next.n);
            });
            if (now.begins && a.out.dstate_in)
                gb.store(a.out.dstate_in + (now.seq * a.in.H + h) * size, dk, dv);
        } else {
            if (now.kind == kState) {
                State<T, DK, DV, FULL> state, entering;
                state.load(whole.before.own, dk, dv, dv, 1);
                entering.load(whole.before.entering, dk, dv, dv, 1);
                to_end<C>(w, l2, now.n);
#pragma unroll
                for (int x = 0; x < state.KT; ++x)
#pragma unroll
                    for (int y = 0; y < state.VT; ++y)
                        state.s[x][y] += entering.s[x][y] * whole.before.fade;
                state.template update<C>(tile_k, tile_v, w, power(l2, (float)now.n));
                state.store(scratch, dk, dv);
            }
            __syncthreads();
        }
        if (next.kind == kNone)
            break;
        if (!AHEAD || now.kind != kTile)
            load(next.t, next.n);
        const bool bad = put();
        now = next;
        if (bad && now.kind == kTile && now.n > 1) {
            whole = now;
            single = now.n - 1;
            now.kind = kNone;
        } else if (now.kind == kTile) {
            --single;
        }
        if (single > 0 && now.kind != kState) {
            next.kind = kState;
            next.t = whole.t;
            next.n = single;
        } else if (single >= 0) {
            next = whole;
            next.t += single;
            next.n = 1;
            next.fresh = whole.fresh && single == whole.n - 1;
            next.begins = whole.begins && single == 0;
            if (single > 0)
                next.before = {scratch, nullptr, 0.f};
        } else {
            single = -1;
            next = step();
        }
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

// The gradients of shared keys and values: the sums over the heads that share them.  The first half of
// the workgroups has the keys', the second the values'.
template <typename T>
__global__ __launch_bounds__(256) void shared_heads_kernel(const AttentionArgs a)
{
    const bool values = blockIdx.x >= gridDim.x / 2;
    const int width = values ? a.in.DV : a.in.DK, KH = a.in.KH, share = a.in.H / KH;
    const float *part = values ? a.part_v : a.part_k;
    T *out = (T *)(values ? a.out.dv : a.out.dk);
    const int64_t ld = values ? a.out.ld_dv : a.out.ld_dk;
    const int64_t per = (int64_t)KH * width, blocks = gridDim.x / 2;
    for (int64_t id = (values ? blockIdx.x - blocks : blockIdx.x) * 256 + threadIdx.x;
         id < a.in.T * per; id += blocks * 256) {
        const int64_t t = id / per;
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
    (void)by_head(in, [&](auto type, auto dk, auto dv, auto full) {
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
        const int marks = (int)attention_marks(a.in, a.cut);
        if (a.cut.joined || marks > 1)  // the first tile has none
            e = launch_attention_ends(a, a.cut.joined, (int)(a.cut.tokens / marks), marks,
                                      stream);
        if (e == hipSuccess)
            e = by_head(a.in, [&](auto type, auto dk, auto dv, auto full) {
                using T = decltype(type);
                constexpr int DK = decltype(dk)::value, DV = decltype(dv)::value;
                return in_launches(a.cut.ranges, a.in.H, [&](int64_t first, dim3 grid) {
                    attention_backward_kernel<T, DK, DV, decltype(full)::value><<<grid, 256, 0, stream>>>(a, first, marks);
                });
            });
        if (e != hipSuccess)
            return e;
        if (a.part_k) {
            const int width = a.in.DK > a.in.DV ? a.in.DK : a.in.DV;
            const int64_t n = (a.in.T * a.in.KH * width + 255) / 256;
            const dim3 grid(2 * (unsigned)(n < 4096 ? n : 4096));
            if (a.in.dt == LBI_BF16)
                shared_heads_kernel<bf16_bits><<<grid, 256, 0, stream>>>(a);
            else
                shared_heads_kernel<float><<<grid, 256, 0, stream>>>(a);
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
