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
// 8 sequences of 2048 tokens, 12 heads of 64, bf16 (101 MB of tokens): 31 us for the walk, 17 for the
// states that ranges add and 6 for the carry.  A walk waits on its chain of products, LDS and
// barriers at three workgroups a CU; the first kernel reads half of what the walk does.  Tiles of 64
// tokens: a state's products cost the same for each token whatever the tile, the tokens' own grow
// with it, and the state's update and barriers are shared by more.
//
// A value that is infinite or NaN would reach earlier tokens of its tile (0 times it is NaN), so
// tiles with one are taken token by token.
#include "lbi_attention.hpp"

namespace lbi {
namespace {

constexpr int C = kAttentionTile;

// Workgroups of a CU that the registers are divided among, by the widths of a key and a value.
template <typename T> constexpr int resident(int widths)
{
    return widths == 256 ? 1 : widths == 192 ? (sizeof(T) == 2 ? 2 : 1) : (sizeof(T) == 2 ? 3 : 2);
}

template <typename T> constexpr int resident_ends(int widths)
{
    return sizeof(T) == 2 || widths == 128 ? resident<T>(widths) : widths == 192 ? 3 : 2;
}

template <typename T, int DK, int DV, bool FULL>
__global__ __launch_bounds__(256, resident<T>(DK + DV)) void attention_kernel(const AttentionArgs a, int64_t first)
{
    constexpr int QS = tile_stride<T>(DK), VS = tile_stride<T>(DV), PS = tile_stride<T>(C);
    __shared__ __align__(16) T tile_q[C * QS], tile_k[C * QS], tile_v[C * VS], tile_p[C * PS];
    __shared__ int flags[4];
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    const int h = blockIdx.x % a.in.H, kh = h / (a.in.H / a.in.KH);
    const int64_t range = first + blockIdx.x / a.in.H;
    const int dk = FULL ? DK : a.in.DK, dv = FULL ? DV : a.in.DV;
    const int64_t size = (int64_t)dk * dv;
    const float l2 = log2_decay(a.in.log_decay, h), scale = a.in.scale;
    const T *q0 = (const T *)a.in.q + h * dk, *k0 = (const T *)a.in.k + kh * dk;
    const T *v0 = (const T *)a.in.v + kh * dv;
    T *o0 = (T *)a.o + h * dv;

    const Sequences seqs = sequences_of(a.in);
    const Rows rows(a, range);
    State<T, DK, DV, FULL> state;
    f4 fade[kCausalTiles<C>];
    causal_fade<C>(fade, l2, scale);
    float w[C / 4];  // what is left of the tile's tokens at its end
    int weights_of = 0;
    // what is left of the state at the tile's first tokens, and 16 tokens on
    const float reach0 = power(l2, (float)(c16 + 1)) * scale, reach16 = power(l2, 16.f);

    TileLoad<T, C, DK, FULL> next_q, next_k;
    TileLoad<T, C, DV, FULL> next_v;
    auto load = [&](int64_t t, int n) {
        next_q.load(q0 + t * a.in.ld_q, a.in.ld_q, n, dk);
        next_k.load(k0 + t * a.in.ld_k, a.in.ld_k, n, dk);
        next_v.load(v0 + t * a.in.ld_v, a.in.ld_v, n, dv);
    };
    auto put = [&] {
        bool bad = next_q.put(tile_q);
        bad |= next_k.put(tile_k);
        bad |= next_v.put(tile_v);
        return any_bad(bad, flags);
    };
    // Tokens t .. t + tokens - 1, whose tiles are in LDS, from the state before them.
    auto work = [&](int64_t t, int tokens) {
        if (tokens != weights_of) {
            to_end<C>(w, l2, tokens);
            weights_of = tokens;
        }
        // p_ij = scale a^(i-j) q_i . k_j, rounded to the tokens' type as an operand: with bf16 the
        // outputs' error against float64 is 0.0018 instead of the 0.0017 that their own rounding is,
        // and a second value of each would double this tile and its products
        causal_tiles<C>([&](int at, int it, int jt) {
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
                    p[r] = lag >= r ? p[r] * fade[at][r] : 0.f;
            }
            put4(tile_p + (16 * it + c16) * PS + 16 * jt + lane_quad<T>(), p);
        });
        __syncthreads();
#pragma unroll
        for (int c = 0; c < DV / 64; ++c) {
            const int col = state.column(c);
            Frag<T> fv[C / 32];
#pragma unroll
            for (int b = 0; b < C / 32; ++b)
                fv[b].cols(tile_v, VS, 32 * b, col);
            Wide<T, 2> fs[DK / 32];  // two: the outputs are rounded to 2^-8 behind it
#pragma unroll
            for (int b = 0; b < DK / 32; ++b)
                pack_tiles(fs[b], state.s[2 * b][c], state.s[2 * b + 1][c]);
            float reach = reach0;
#pragma unroll 2
            for (int it = 0; it < C / 16; ++it) {
                f4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int b = 0; b < DK / 32; ++b) {
                    Frag<T> fq;
                    fq.rows(tile_q, QS, 16 * it, 32 * b);
                    mma(o, fs[b], fq);
                }
                o *= reach;
                reach *= reach16;
#pragma unroll
                for (int b = 0; b < C / 32; ++b)
                    if (b <= it / 2) {
                        Frag<T> fp;
                        fp.rows(tile_p, PS, 16 * it, 32 * b);
                        mma(o, fv[b], fp);
                    }
                const int i = 16 * it + c16;
                if (i < tokens)
                    store4<T, FULL>(o0 + (t + i) * a.ld_o + col + 4 * g, dv - col - 4 * g, o);
            }
        }
        phase();
        state.template update<C>(tile_k, tile_v, w, power(l2, (float)tokens));
    };
    // Tiles of the range, in order: rows t .. t + n - 1 of one sequence.
    Segment seg;
    seg.enter(seqs, rows.first, true);
    const bool starts_here = seg.start >= rows.first;
    struct Item {
        int64_t t, seq;
        int n;  // 0: none
        bool first, last, behind;  // of its sequence's tiles in the range; the sequence leaves it
    };
    auto item = [&](int64_t t, bool first) -> Item {
        const int64_t stop = seg.end < rows.end ? seg.end : rows.end;
        const int n = stop - t < C ? (int)(stop - t) : C;
        return {t, seg.seq, n, first, t + n == seg.end, seg.end > rows.end};
    };
    Item now = {}, next = item(rows.first, true);
    while (true) {
        if (next.n > 0)
            load(next.t, next.n);  // on its way while the tile in LDS is worked on
        if (now.n > 0) {
            if (now.first) {
                const float *p = nullptr;
                if (now.t == rows.first && !starts_here)
                    p = a.ends + ((range - 1) * a.in.H + h) * size;
                else if (a.starts && now.behind)  // another workgroup may have written the slot
                    p = a.starts + (range * a.in.H + h) * size;
                else if (a.in.state_in) {
                    const int64_t row = state_row(a.slots, a.n_slots, now.seq);
                    p = row >= 0 ? a.in.state_in + (row * a.in.H + h) * size : nullptr;
                }
                state.load(p, dk, dv, dv, 1);
            }
            work(now.t, now.n);
            if (now.last && a.state_out) {
                const int64_t row = state_row(a.slots, a.n_slots, now.seq);
                if (row >= 0)
                    state.store(a.state_out + (row * a.in.H + h) * size, dk, dv);
            }
        }
        __syncthreads();
        if (next.n == 0)
            return;
        if (put() && next.n > 1) {  // a token by itself
            next.n = 1;
            next.last = next.t + 1 == seg.end;
            now.n = 0;
            continue;
        }
        now = next;
        const int64_t t = now.t + now.n;
        if (t >= rows.end) {
            next.n = 0;
        } else {
            if (now.last)
                seg.advance(seqs);
            next = item(t, now.last);
        }
    }
}

// What a range adds to the state of the sequence that passes its end, or (backward) to the gradient
// of the state of the sequence that passes its start.  With marks (the gradient's), also what the
// range, or the sequence's first state, adds to the states before the second and further tiles of
// each of its sequences.
// both: every second workgroup goes backward, otherwise none does.
template <typename T, int DK, int DV, bool FULL>
__global__ __launch_bounds__(256, resident_ends<T>(DK + DV)) void ends_kernel(const AttentionArgs a,
                                                                        int64_t first, bool both,
                                                                        int mark_rows, int every)
{
    // Half a tile of float32 at 128 keys or values, of which the registers hold three workgroups a CU
    // instead of one: 732 of them took 53 us, and 28 so.  (64 and 64: 59, and 64 so.)
    constexpr int C = sizeof(T) == 4 && DK + DV >= 192 ? 32 : kAttentionTile;
    constexpr int QS = tile_stride<T>(DK), VS = tile_stride<T>(DV);
    __shared__ __align__(16) T tile_a[C * QS], tile_b[C * VS];
    const int h = blockIdx.x % a.in.H, kh = h / (a.in.H / a.in.KH);
    const int64_t id = first + blockIdx.x / a.in.H, range = both ? id >> 1 : id;
    const bool backward = both && (id & 1);
    const int marks = backward ? 0 : every, tile_rows = marks > 0 ? mark_rows : C;
    const int dk = FULL ? DK : a.in.DK, dv = FULL ? DV : a.in.DV;
    const int64_t size = (int64_t)dk * dv, at = range * a.in.H + h;
    const float l2 = log2_decay(a.in.log_decay, h);
    const Sequences seqs = sequences_of(a.in);
    const Rows rows(a, range);
    const T *a0 = backward ? (const T *)a.in.q + h * dk : (const T *)a.in.k + kh * dk;
    const T *b0 = backward ? (const T *)a.dout + h * dv : (const T *)a.in.v + kh * dv;
    const int64_t ld_a = backward ? a.in.ld_q : a.in.ld_k;
    const int64_t ld_b = backward ? a.ld_dout : a.in.ld_v;
    State<T, DK, DV, FULL> state;
    float w[C / 4];
    int weights_of = 0;
    TileLoad<T, C, DK, FULL> next_a;
    TileLoad<T, C, DV, FULL> next_b;
    Segment seg;
    seg.enter(seqs, backward || marks > 0 ? rows.first : rows.end - 1, true);
    while (true) {
        const bool before = seg.start < rows.first, behind = seg.end > rows.end;
        const int64_t from = before ? rows.first : seg.start, to = behind ? rows.end : seg.end;
        // one sequence passes the end, or the start; of others nothing but their marks is kept
        const bool passes = a.cut.joined && (backward ? before : behind);
        if (passes && h == 0 && threadIdx.x == 0)
            (backward ? a.head_flags : a.end_flags)[range] = before && behind ? kWhole : kPart;
        const float *begin = nullptr;
        if (backward) {
            if (!behind && a.dstate_out)
                begin = a.dstate_out + (seg.seq * a.in.H + h) * size;
        } else if (!before && a.in.state_in) {
            const int64_t row = state_row(a.slots, a.n_slots, seg.seq);
            begin = row >= 0 ? a.in.state_in + (row * a.in.H + h) * size : nullptr;
        }
        // the last tile is for what passes only
        const int tiles = (int)((to - from + tile_rows - 1) / tile_rows) - (passes ? 0 : 1);
        if (tiles > 0) {
            state.load(begin, dk, dv, dv, 1);
            if (a.starts && passes && !before)
                state.store(a.starts + at * size, dk, dv);
            int n = 0;
            int64_t t = 0;
            auto load = [&](int i) {
                t = from + (int64_t)(backward ? tiles - 1 - i : i) * tile_rows;
                n = to - t < tile_rows ? (int)(to - t) : tile_rows;
                next_a.load(a0 + t * ld_a, ld_a, n, dk);
                next_b.load(b0 + t * ld_b, ld_b, n, dv);
            };
            load(0);
            for (int i = 0; i < tiles; ++i) {
                next_a.put(tile_a);
                next_b.put(tile_b);
                __syncthreads();
                const int tokens = n;
                const int64_t end = t + n;
                if (i + 1 < tiles)
                    load(i + 1);
                if (tokens != weights_of) {
                    if (backward)
                        from_start<C>(w, l2, tokens, a.in.scale);
                    else
                        to_end<C>(w, l2, tokens);
                    weights_of = tokens;
                }
                state.template update<C>(tile_a, tile_b, w, power(l2, (float)tokens));
                if (marks > 0 && end < to)
                    state.store(a.marks + (at * marks + (end - rows.first) / tile_rows - 1) * size,
                                dk, dv);
                __syncthreads();
            }
            if (passes)
                state.store((backward ? a.heads : a.ends) + at * size, dk, dv);
        }
        if (!passes && a.cut.joined && h == 0 && threadIdx.x == 0 &&
            (backward || seg.end >= rows.end))
            (backward ? a.head_flags : a.end_flags)[range] = 0;
        if (marks == 0 || to >= rows.end)
            return;
        seg.advance(seqs);
    }
}

// States along the ranges of a sequence (of all tokens, with offsets), or their gradients against
// them: one thread for V neighbouring values of a head, which lie at a multiple of V floats.
template <int V>
__global__ __launch_bounds__(256) void carry_kernel(const AttentionArgs a, int64_t first,
                                                    int blocks, bool both)
{
    typedef float fv __attribute__((ext_vector_type(V)));
    const int64_t size = (int64_t)a.in.DK * a.in.DV;
    const uint32_t id = blockIdx.x;
    const int64_t e = ((int64_t)(id % blocks) * 256 + threadIdx.x) * V;
    const int h = id / blocks % a.in.H;
    const int64_t which = first + id / blocks / a.in.H, chain = both ? which >> 1 : which;
    const bool backward = both && (which & 1);
    if (e >= size)
        return;
    const int64_t count = a.cut.per_sequence > 0 ? a.cut.per_sequence : a.cut.ranges;
    const float fade = power(log2_decay(a.in.log_decay, h), (float)a.cut.tokens);
    float *p = (backward ? a.heads : a.ends) + h * size + e;
    const int32_t *flags = backward ? a.head_flags : a.end_flags;
    const int64_t step = a.in.H * size;
    const int64_t last = backward ? 0 : count - 1, way = backward ? -1 : 1;
    float *at = p + (chain * count + (count - 1 - last)) * step;
    flags += chain * count + (count - 1 - last);
    // the next ranges are on their way before this step's stores, whether something passes them or not
    constexpr int AHEAD = V == 4 ? 4 : 8;
    fv v = 0.f, next[AHEAD];
    int32_t next_flag[AHEAD];
    auto load = [&](int64_t done) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int64_t to = (done + k < count ? done + k : count - 1) * way;
            next_flag[k] = flags[to];
            next[k] = *(const fv *)(at + to * step);
        }
    };
    load(0);
    for (int64_t done = 0; done < count; done += AHEAD) {
        fv x[AHEAD];
        int32_t f[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            x[k] = next[k];
            f[k] = next_flag[k];
        }
        if (done + AHEAD < count)
            load(done + AHEAD);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            v = f[k] == kWhole ? x[k] + fade * v : x[k];
            if (f[k] == kWhole && done + k < count)
                *(fv *)(at + (done + k) * way * step) = v;
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
    if (from)
        from += (row * a.in.H + h) * size;
    constexpr int MOST = LBI_ATTENTION_MAX_DIM * LBI_ATTENTION_MAX_DIM / 2048;
    float x[MOST][8];
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        const int e = (i * 256 + threadIdx.x) * 8;
        load_some<8>(from + (e < size ? e : 0), from ? (int)size - e : 0, x[i]);
    }
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        const int e = (i * 256 + threadIdx.x) * 8;
        store_some<8>(to + (e < size ? e : 0), (int)size - e, x[i]);
    }
}

// One token: a workgroup takes a head of a sequence, COLS lanes of 4 columns side by side, the
// other lanes further rows.  Bound by the state, which is read and written once: 64 sequences, 12 heads
// of 64 and 128, 50 MB, take 11 us (a copy of that total 7.5).
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

// The tokens of a range: the fewest tile times of
//
//   rounds (tiles + 2) + [cut: rounds' (tiles + 2) / 2 + 3 + ranges of a sequence / 32]
//
// for the forward pass, where a round is what the GPU holds at once, a workgroup costs two tiles
// besides its own, forming the states that ranges add takes half of a walk with outputs, and
// carrying them three tile times and more for each 32 ranges; the gradient's walk counts twice, and
// the states before it are formed for both sides at once.  Measured against ranges of 64 to 1024
// tokens, 12 gradients of 2271 to 31948 tokens: within 7 per cent of the best of them, one (36 heads
// of 16, three sequences) 12.  Forward, bf16 and float32: within 8.
AttentionCut attention_cut(const lbi_attention_inputs &in, bool ragged, bool backward)
{
    AttentionCut best = {};
    if (in.T == 0)
        return best;
    const int widths = (in.DK <= 64 ? 64 : 128) + (in.DV <= 64 ? 64 : 128);
    const bool bf16 = in.dt == LBI_BF16;
    const int64_t ends_slots = 256 * (bf16 ? resident_ends<bf16_bits>(widths) : resident_ends<float>(widths));
    const int64_t slots = backward ? (widths <= (bf16 ? 128 : 192) ? 512 : 256)
                                   : 256 * (bf16 ? resident<bf16_bits>(widths) : resident<float>(widths));
    const int64_t len = ragged ? in.T : in.T / in.sequences;
    const int64_t most = (len + kAttentionTile - 1) / kAttentionTile;
    double least = 0;
    for (int64_t tiles = 1;; ++tiles) {
        if (tiles > 64 && tiles < most)
            tiles = most;  // the whole of it
        AttentionCut c = {};
        c.tokens = tiles * kAttentionTile;
        const int64_t per = (len + c.tokens - 1) / c.tokens;
        c.ranges = ragged ? per : per * in.sequences;
        c.per_sequence = ragged ? 0 : (int32_t)per;
        c.joined = per > 1;
        const double groups = (double)c.ranges * in.H;
        auto rounds = [&](double groups, int64_t n) {
            return (double)((int64_t)((groups + n - 1) / n)) * (double)(tiles + 2);
        };
        const double walk = rounds(groups, slots), ends = rounds(groups, ends_slots) / 2;
        const double join = 3 + (double)per / 32;
        const double cost = !backward    ? walk + (c.joined ? ends + join : 0)
                            : !c.joined ? 2 * walk + ends
                                        : 2 * walk + rounds(2 * groups, ends_slots) / 2 + join;
        if (tiles == 1 || cost < least) {
            least = cost;
            best = c;
        }
        if (tiles >= most)
            return best;
    }
}

// Both sides of the gradient go in one launch, which fills the GPU better than one after the other:
// 46 us instead of 52 (8 sequences of 2048 tokens, 12 heads of 64, bf16).
hipError_t launch_attention_ends(const AttentionArgs &a, bool both, int mark_rows, int marks,
                                 hipStream_t stream)
{
    const int64_t sides = both ? 2 : 1;
    hipError_t e = by_head(a.in, [&](auto type, auto dk, auto dv, auto full) {
        return in_launches(a.cut.ranges * sides, a.in.H, [&](int64_t first, dim3 grid) {
            ends_kernel<decltype(type), decltype(dk)::value, decltype(dv)::value,
                        decltype(full)::value>
                <<<grid, 256, 0, stream>>>(a, first, both, mark_rows, marks);
        });
    });
    if (e != hipSuccess || !a.cut.joined)
        return e;
    const int64_t size = (int64_t)a.in.DK * a.in.DV;
    const int64_t chains = (a.cut.per_sequence > 0 ? a.in.sequences : 1) * sides;
    // four values to a thread where that leaves each CU its 256: 96 chains of 4 or 5 states of 4096
    // values take 6 us so, 10 one by one; 12 chains of about 200 took 16, one by one 9
    const bool wide = size % 4 == 0 && chains * a.in.H * (size / 4) >= 256 * 256;
    const int blocks = (int)((size / (wide ? 4 : 1) + 255) / 256);
    return in_launches(chains, (int64_t)blocks * a.in.H, [&](int64_t first, dim3 grid) {
        if (wide) carry_kernel<4><<<grid, 256, 0, stream>>>(a, first, blocks, both);
        else carry_kernel<1><<<grid, 256, 0, stream>>>(a, first, blocks, both);
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
            e = launch_attention_ends(a, false, 0, 0, stream);
        if (e == hipSuccess)
            e = by_head(a.in, [&](auto type, auto dk, auto dv, auto full) {
                return in_launches(a.cut.ranges, a.in.H, [&](int64_t first, dim3 grid) {
                    attention_kernel<decltype(type), decltype(dk)::value, decltype(dv)::value,
                        decltype(full)::value>
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
