// Short causal convolution along packed sequences, channel by channel: forward,
// gradient, and one token a sequence.
//
// A thread owns V consecutive channels and a run of tokens, which it takes in pieces
// of up to PIECE tokens of one sequence.  All rows of a piece and the W - 1 before it
// are loaded at once, so that some twenty loads of a thread are in flight, and
// everything else happens in registers.  The bytes are the tensors' own (the rows
// around a piece come from cache), a few operations for each: the bound is HBM.
// Lanes of a workgroup lie along the channels (a row's values are contiguous) and,
// above that, along the runs.
//
// Measured, four taps, bf16, 1536 channels: 8201 packed tokens of 13 sequences, 51 MB, in
// 14.5 us (3.5 TB/s; a copy of as many bytes 8.4 us); the gradient of 16384 tokens, 151 MB,
// in 35 + 4 us (3.9 TB/s); one token of 64 sequences 5.3 us, dependent trips to memory.
#include "lbi_block.hpp"

namespace lbi {
namespace {

constexpr int64_t kThreads = 1 << 18;  // threads wanted in all: 16 wavefronts a CU
constexpr int kPiece = 16;
template <typename T> constexpr int backward_piece_rows() { return 32 / sizeof(T); }

// How a [tokens][channels] plane is cut: lanes along the channels (a power of
// two), runs beside them in a workgroup of 256, and tokens a run.
struct Cut {
    int lanes, runs, tokens;
    int64_t row_blocks;
    int32_t col_blocks;
};
Cut cut_of(int64_t T, int32_t D, int V, int most)
{
    const int64_t vec = (D + V - 1) / V;
    int lanes = 1;
    while (lanes < 64 && lanes < vec)
        lanes *= 2;
    int tokens = 4;
    while (tokens < most && T * vec > (int64_t)tokens * kThreads)
        tokens *= 2;
    const int runs = 256 / lanes;
    const int64_t per = (int64_t)runs * tokens;
    return {lanes, runs, tokens, (T + per - 1) / per,
            (int32_t)((vec + lanes - 1) / lanes)};
}
// Two channels a lane: the rows in flight and, in the gradient, its sums then leave
// room for four wavefronts a SIMD, which the operations need.  16384 tokens, 1536 channels,
// bf16: forward 19 us (eight channels a lane 24), gradient 35 (four channels 46).
constexpr int kWidth = 2;
Cut forward_cut(int64_t T, int32_t D) { return cut_of(T, D, kWidth, kPiece); }
Cut backward_cut(int64_t T, int32_t D) { return cut_of(T, D, kWidth, 512); }

// The last vector of a row whose width is no multiple of V moves back to end with
// the row: some channels are then computed twice, to the same values, and no lane
// works on a part of a vector (unless the row is shorter than one).
template <int V> __device__ __forceinline__ void whole_vector(int32_t D, int *d, int *left)
{
    if (*left < V && D >= V) {
        *d = D - V;
        *left = V;
    }
}

// Row i of the rows from p on, or the last one that is there: a load that no lane has
// to skip.  (Row strides are limited, so the distance fits 32 bits.)
template <typename T>
__device__ __forceinline__ const T *row_at(const T *p, int i, int there, uint32_t bytes)
{
    return (const T *)((const char *)p + (uint64_t)(uint32_t)(i < there ? i : there) * bytes);
}

// V values of a row: all of them (FULL), or the first `left`.
template <bool FULL, int V, typename T>
__device__ __forceinline__ void load_row(const T *p, int left, Raw<T, V> &r)
{
    if constexpr (FULL) {
        r.load(p, V);
    } else {
        // a row narrower than a vector: the values that are not there repeat the first
        T v[V];
#pragma unroll
        for (int i = 0; i < V; ++i)
            v[i] = p[i < left ? i : 0];
        __builtin_memcpy(&r, v, sizeof(r));
    }
}
template <bool FULL, int V, typename T>
__device__ __forceinline__ void store_row(T *p, int left, const float (&v)[V])
{
    if constexpr (FULL)
        store_all<V>(p, v);
    else
        store_some<V>(p, left, v);
}

// The taps of V channels, weight[d][w] -> k[w][i].
template <int W, int V>
__device__ __forceinline__ void load_taps(const float *weight, int d, int left, float (&k)[W][V])
{
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int w = 0; w < W; ++w)
            k[w][i] = i < left ? weight[(int64_t)(d + i) * W + w] : 0.f;
}

// The W - 1 rows of x before row t, oldest first, ahead of knowing whose they are...
template <int W, int V, typename T>
__device__ __forceinline__ void load_rows_before(const ConvArgs &a, int64_t t, int d, int left,
                                                 Raw<T, V> (&before)[W - 1])
{
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int64_t row = t - (W - 1) + j;
        before[j].load((const T *)a.x + d + (row > 0 ? row : 0) * a.ld_x, left);
    }
}
// ... and the W - 1 tokens before row t of its sequence: these, or rows of the state
// where the sequence has not that many.
template <int W, int V, typename T>
__device__ __forceinline__ void window_of(const ConvArgs &a, const Segment &seg, int64_t t, int d,
                                          int left, const Raw<T, V> (&before)[W - 1],
                                          float (&win)[W - 1][V])
{
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        before[j].unpack(win[j]);
    if (t - seg.start >= W - 1)
        return;
    const int64_t slot = a.state_in ? state_row(a.slots, a.n_slots, seg.seq) : -1;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int64_t row = t - (W - 1) + j, k = (W - 1) + (row - seg.start);
        if (row < seg.start)
            load_some<V>((const T *)a.state_in + (slot < 0 ? 0 : (slot * (W - 1) + k) * a.D + d),
                         slot < 0 ? 0 : left, win[j]);
    }
}

// The state after sequence s: the last W - 1 of its old state and its tokens.
template <int W, int V, typename T>
__device__ __forceinline__ void write_state(const ConvArgs &a, const Sequences &q, int64_t s, int d,
                                            int left)
{
    const int64_t slot = state_row(a.slots, a.n_slots, s);
    if (slot < 0)
        return;
    const int64_t start = q.at(s), len = q.at(s + 1) - start;
    float v[W - 1][V];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int64_t p = len - (W - 1) + j;
        if (p >= 0)
            load_some<V>((const T *)a.x + (start + p) * a.ld_x + d, left, v[j]);
        else if (a.state_in && len >= 0)
            load_some<V>((const T *)a.state_in + (slot * (W - 1) + len + j) * a.D + d, left, v[j]);
        else
            load_some<V>((const T *)a.x, 0, v[j]);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        store_some<V>((T *)a.state_out + (slot * (W - 1) + j) * a.D + d, left, v[j]);
}

// A run, piece by piece.  UNIFORM: by a wavefront whose lanes all have the same run, so
// that rows have uniform addresses.
template <int W, int V, bool FULL, bool UNIFORM, typename T>
__device__ __forceinline__ void conv_run(const ConvArgs &a, const Sequences &q, int64_t t0,
                                         int64_t t1, int d, int left)
{
    const int64_t last = a.T - 1;
    const uint32_t lane = (uint32_t)d * sizeof(T), bytes = (uint32_t)(a.ld_x * (int64_t)sizeof(T));
    Raw<T, V> rows[kPiece], before[W - 1];
    float k[W][V], bias[V];
    if constexpr (UNIFORM) {
        t0 = uniform(t0);
        t1 = uniform(t1);
    }
    auto load = [&](int64_t t) {
        const T *p = (const T *)a.x + t * a.ld_x;
        const int there = (int)(last - t < kPiece ? last - t : kPiece);
        if constexpr (UNIFORM) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                const int64_t row = t - (W - 1) + j;
                before[j].load(lane_address((const T *)a.x + (row > 0 ? row : 0) * a.ld_x, lane), V);
            }
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                rows[i].load(lane_address(p + (i < there ? i : there) * a.ld_x, lane), V);
        } else {
            load_rows_before<W, V, T>(a, t, d, left, before);
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                load_row<FULL, V>(row_at(p + d, i, there, bytes), left, rows[i]);
        }
    };
    load(t0);  // the first rows are known before their sequence is
    load_taps<W, V>(a.weight, d, left, k);
    load_some<V>(a.bias ? a.bias + d : a.bias, a.bias ? left : 0, bias);
    Segment seg;
    seg.enter(q, t0, UNIFORM);
    for (int64_t t = t0;;) {
        int64_t end = seg.end < t1 ? seg.end : t1;
        end = end < t + kPiece ? end : t + kPiece;
        const int n = (int)(end - t);
        float win[W - 1][V];
        window_of<W, V, T>(a, seg, t, d, left, before, win);
        T *out = (T *)a.out + t * a.ld_out;
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            float cur[V], y[V];
            rows[i].unpack(cur);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float v = bias[e];
#pragma unroll
                for (int w = 0; w < W - 1; ++w)
                    v += k[w][e] * win[w][e];
                v += k[W - 1][e] * cur[e];
                y[e] = a.silu ? silu(v) : v;
#pragma unroll
                for (int w = 0; w < W - 2; ++w)
                    win[w][e] = win[w + 1][e];
                win[W - 2][e] = cur[e];
            }
            if (i < n)
                store_row<FULL, V>(lane_address(out + i * a.ld_out, lane), left, y);
        }
        t = end;
        if (t >= t1)
            break;
        if (t == seg.end)
            seg.advance(q);
        load(t);
    }
}

// Row blocks from `first` on: those below row_blocks convolve, the others write states.
template <int W, typename T>
__global__ __launch_bounds__(256) void conv_kernel(const ConvArgs a, const Cut c, int64_t first)
{
    constexpr int V = kWidth;
    const Sequences q = {a.offsets, a.T, a.B, a.B > 0 ? a.T / a.B : 0};
    const unsigned row_of = blockIdx.x / (unsigned)c.col_blocks;
    const int col_block = (int)(blockIdx.x - row_of * c.col_blocks);
    int d = (col_block * c.lanes + (int)threadIdx.x % c.lanes) * V, left = a.D - d;
    if (left <= 0)
        return;
    const int64_t block = first + row_of;
    const int64_t run = block * c.runs + threadIdx.x / c.lanes;
    if (block >= c.row_blocks) {
        const int64_t s = run - c.row_blocks * c.runs;
        if (s < a.B)
            write_state<W, V, T>(a, q, s, d, left);
        return;
    }
    const int64_t t0 = run * c.tokens, t1 = t0 + c.tokens < a.T ? t0 + c.tokens : a.T;
    if (t0 >= t1)
        return;
    whole_vector<V>(a.D, &d, &left);
    // a wavefront along the channels has one run, unless the channels end in it
    if (left < V)
        conv_run<W, V, false, false, T>(a, q, t0, t1, d, left);
    else if (c.lanes == 64 && __popcll(__ballot(true)) == 64)
        conv_run<W, V, true, true, T>(a, q, t0, t1, d, left);
    else
        conv_run<W, V, true, false, T>(a, q, t0, t1, d, left);
}

template <int W, typename T>
__global__ __launch_bounds__(256) void conv_step_kernel(const ConvArgs a, int64_t first)
{
    constexpr int V = 16 / sizeof(T);
    const int64_t vec = (a.D + V - 1) / V;
    const int64_t id = (first + blockIdx.x) * 256 + threadIdx.x;
    const int64_t row = id / vec;
    const int d = (int)(id - row * vec) * V, left = a.D - d;
    if (row >= a.T)
        return;
    const int64_t slot = state_row(a.slots, a.n_slots, row);
    float k[W][V], v[W][V], y[V];
    load_some<V>((const T *)a.x + row * a.ld_x + d, left, v[W - 1]);
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        load_some<V>((const T *)a.state_in + ((slot < 0 ? 0 : slot) * (W - 1) + j) * a.D + d,
                     slot < 0 ? 0 : left, v[j]);
    load_taps<W, V>(a.weight, d, left, k);
    load_some<V>(a.bias ? a.bias + d : a.bias, a.bias ? left : 0, y);
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int w = 0; w < W; ++w)
            y[i] += k[w][i] * v[w][i];
        y[i] = a.silu ? silu(y[i]) : y[i];
    }
    store_some<V>((T *)a.out + row * a.ld_out + d, left, y);
    if (slot >= 0)
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            store_some<V>((T *)a.state_out + (slot * (W - 1) + j) * a.D + d, left, v[j + 1]);
}

// Gradient of a piece: with v the convolution and dv = dout f'(v), token t receives
// dx_t = sum_j dv_{t+j} weight_{W-1-j} over the tokens t + j of its sequence, and its old
// state the same of the tokens that read it.
//
// Rows t .. t + n - 1 of one sequence, all rows loaded at once; dv is formed for the W - 1
// rows after them too.  Neither the old nor the new state takes part.  WHOLE: a full
// piece well within its sequence, the same for all lanes of the wavefront, so that rows
// have uniform addresses and nothing is chosen by lane.
template <int W, int V, bool WHOLE, typename T>
__device__ __forceinline__ void backward_piece(const ConvArgs &a, const Segment &seg, int64_t t,
                                               int n, int d, const float (&k)[W][V],
                                               const float (&bias)[V], float (&sums)[W + 1][V])
{
    constexpr int PIECE = backward_piece_rows<T>(), ROWS = PIECE + W - 1;
    Raw<T, V> rx[ROWS], ry[ROWS], before[W - 1];
    const uint32_t lane = (uint32_t)d * sizeof(T);
    if constexpr (WHOLE) {
        t = uniform(t);
        const T *px = (const T *)a.x + t * a.ld_x, *py = (const T *)a.dout + t * a.ld_dout;
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            before[j].load(lane_address(px - (W - 1 - j) * a.ld_x, lane), V);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            rx[i].load(lane_address(px + i * a.ld_x, lane), V);
            ry[i].load(lane_address(py + i * a.ld_dout, lane), V);
        }
    } else {
        const int64_t last = a.T - 1;
        const int there = (int)(last - t < ROWS ? last - t : ROWS);
        const uint32_t bx = (uint32_t)(a.ld_x * (int64_t)sizeof(T));
        const uint32_t by = (uint32_t)(a.ld_dout * (int64_t)sizeof(T));
        const T *px = (const T *)a.x + t * a.ld_x + d, *py = (const T *)a.dout + t * a.ld_dout + d;
        load_rows_before<W, V, T>(a, t, d, V, before);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            rx[i].load(row_at(px, i, there, bx), V);
            ry[i].load(row_at(py, i, there, by), V);
            if (i % 4 == 3)  // (the addresses of all rows at once would take the registers)
                __builtin_amdgcn_sched_barrier(0);
        }
    }
    float win[W - 1][V], dv[W][V];  // dv: of the last W rows, the newest last
    if constexpr (WHOLE) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            before[j].unpack(win[j]);
    } else {
        window_of<W, V, T>(a, seg, t, d, V, before, win);
    }
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
        for (int e = 0; e < V; ++e)
            dv[w][e] = 0.f;
    const int reach = seg.end - t < ROWS ? (int)(seg.end - t) : ROWS;  // rows of the sequence
    T *out = (T *)a.out + t * a.ld_out;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        __builtin_amdgcn_sched_barrier(0);  // one row's values widened at a time
        float cx[V], cy[V], whole[V];
        rx[i].unpack(cx);
        ry[i].unpack(cy);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float v = bias[e];
#pragma unroll
            for (int w = 0; w < W - 1; ++w)
                v += k[w][e] * win[w][e];
            v += k[W - 1][e] * cx[e];
            float g = cy[e];
            if (a.silu)
                g *= silu_slope(v, sigmoid(v));
            if (!WHOLE)
                g = i < reach ? g : 0.f;
            if (i < PIECE) {
                const float mine = WHOLE || i < n ? g : 0.f;
#pragma unroll
                for (int w = 0; w < W - 1; ++w)
                    sums[w][e] += mine * win[w][e];
                sums[W - 1][e] += mine * cx[e];
                sums[W][e] += mine;
#pragma unroll
                for (int w = 0; w <= W; ++w)
                    pin(sums[w][e]);
            }
#pragma unroll
            for (int w = 0; w < W - 1; ++w)
                dv[w][e] = dv[w + 1][e];
            dv[W - 1][e] = g;
#pragma unroll
            for (int w = 0; w < W - 2; ++w)
                win[w][e] = win[w + 1][e];
            win[W - 2][e] = cx[e];
            // row i - (W - 1), which is now whole
            whole[e] = dv[0][e] * k[W - 1][e];
#pragma unroll
            for (int j = 1; j < W; ++j)
                whole[e] += dv[j][e] * k[W - 1 - j][e];
        }
        const int r = i - (W - 1);
        if (r >= 0 && (WHOLE || r < n))
            store_all<V>(lane_address(out + r * a.ld_out, lane), whole);
    }
}

// The same token by token, for any piece: the old state's gradient where the piece
// begins with its sequence, the new state's where it holds tokens of it, and the
// first `left` channels only.  (Rows a sequence's ends touch, and rows narrower
// than a vector.)
template <int W, int V, typename T>
__device__ __forceinline__ void backward_edge(const ConvArgs &a, const Segment &seg, int64_t t, int n,
                                           int d, int left, const float (&k)[W][V],
                                           const float (&bias)[V], float (&sums)[W + 1][V])
{
    const T *x = (const T *)a.x + d, *dy = (const T *)a.dout + d;
    T *dx = (T *)a.out + d;
    const int64_t len = seg.end - seg.start, state = seg.seq * (W - 1);
    Raw<T, V> before[W - 1];
    load_rows_before<W, V, T>(a, t, d, left, before);
    float win[W - 1][V], dv[W][V];
    window_of<W, V, T>(a, seg, t, d, left, before, win);
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
        for (int e = 0; e < V; ++e)
            dv[w][e] = 0.f;
#pragma unroll 1
    for (int i = 0; i < n + W - 1; ++i) {
        const bool there = t + i < seg.end;
        float cx[V], cy[V], whole[V];
        load_some<V>(x + (there ? (t + i) * a.ld_x : 0), there ? left : 0, cx);
        load_some<V>(dy + (there ? (t + i) * a.ld_dout : 0), there ? left : 0, cy);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float v = bias[e];
#pragma unroll
            for (int w = 0; w < W - 1; ++w)
                v += k[w][e] * win[w][e];
            v += k[W - 1][e] * cx[e];
            float g = cy[e];
            if (a.silu)
                g *= silu_slope(v, sigmoid(v));
            g = there ? g : 0.f;
            const bool mine = there && i < n;
#pragma unroll
            for (int w = 0; w < W - 1; ++w)
                sums[w][e] += mine ? g * win[w][e] : 0.f;
            sums[W - 1][e] += mine ? g * cx[e] : 0.f;
            sums[W][e] += mine ? g : 0.f;
#pragma unroll
            for (int w = 0; w < W - 1; ++w)
                dv[w][e] = dv[w + 1][e];
            dv[W - 1][e] = g;
#pragma unroll
            for (int w = 0; w < W - 2; ++w)
                win[w][e] = win[w + 1][e];
            win[W - 2][e] = cx[e];
            whole[e] = 0.f;
#pragma unroll
            for (int j = 0; j < W; ++j)
                whole[e] += dv[j][e] * k[W - 1 - j][e];
        }
        // Row i - (W - 1) of the piece is whole, as row `p` of the old state followed
        // by the sequence, of which the last W - 1 rows are the new state.
        const int r = i - (W - 1);
        const int64_t p = (W - 1) + (t + r - seg.start);
        if ((r < 0 && (t != seg.start || !a.state_out)) || r >= n)
            continue;
        if (a.dstate_out && p >= len) {
            float o[V];
            load_some<V>((const T *)a.dstate_out + (state + p - len) * a.D + d, left, o);
#pragma unroll
            for (int e = 0; e < V; ++e)
                whole[e] += o[e];
        }
        T *to = r < 0 ? (T *)a.state_out + (state + p) * a.D + d : dx + (t + r) * a.ld_out;
        store_some<V>(to, left, whole);
    }
}

template <int W, typename T>
__global__ __launch_bounds__(256) void conv_backward_kernel(const ConvArgs a, const Cut c,
                                                            int64_t first)
{
    constexpr int V = kWidth;
    const Sequences q = {a.offsets, a.T, a.B, a.B > 0 ? a.T / a.B : 0};
    const unsigned row_of = blockIdx.x / (unsigned)c.col_blocks;
    const int col_block = (int)(blockIdx.x - row_of * c.col_blocks);
    const int64_t block_of = first + row_of;
    int d = (col_block * c.lanes + (int)threadIdx.x % c.lanes) * V, left = a.D - d;
    const int64_t run = block_of * c.runs + threadIdx.x / c.lanes;
    if (block_of >= c.row_blocks) {
        // the states of empty sequences pass through
        const int64_t s = run - c.row_blocks * c.runs;
        if (left <= 0 || s >= a.B || q.at(s + 1) > q.at(s))
            return;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            float v[V];
            const int64_t at = (s * (W - 1) + j) * a.D + d;
            load_some<V>((const T *)a.dstate_out + (a.dstate_out ? at : 0), a.dstate_out ? left : 0, v);
            store_some<V>((T *)a.state_out + at, left, v);
        }
        return;
    }
    const bool live = left > 0;
    if (live)
        whole_vector<V>(a.D, &d, &left);
    const int64_t t0 = run * c.tokens, t1 = t0 + c.tokens < a.T ? t0 + c.tokens : a.T;
    float sums[W + 1][V];  // dweight, dbias
#pragma unroll
    for (int w = 0; w <= W; ++w)
#pragma unroll
        for (int i = 0; i < V; ++i)
            sums[w][i] = 0.f;
    if (live && t0 < t1) {
        float k[W][V], bias[V];
        load_taps<W, V>(a.weight, d, left, k);
        load_some<V>(a.bias ? a.bias + d : a.bias, a.bias ? left : 0, bias);
        Segment seg;
        // a wavefront along the channels has one run, unless the channels end in it
        constexpr int PIECE = backward_piece_rows<T>();
        const bool together = c.lanes == 64 && __popcll(__ballot(true)) == 64;
        seg.enter(q, t0, together);
        for (int64_t t = t0; t < t1;) {
            int64_t end = seg.end < t1 ? seg.end : t1;
            end = end < t + PIECE ? end : t + PIECE;
            const bool edge = left < V || (a.state_out && t == seg.start) ||
                              (a.dstate_out && end > seg.end - (W - 1));
            const bool whole = together && end - t == PIECE && t - seg.start >= W - 1 &&
                               seg.end - t >= PIECE + W - 1;
            if (edge)
                backward_edge<W, V, T>(a, seg, t, (int)(end - t), d, left, k, bias, sums);
            else if (whole)
                backward_piece<W, V, true, T>(a, seg, t, (int)(end - t), d, k, bias, sums);
            else
                backward_piece<W, V, false, T>(a, seg, t, (int)(end - t), d, k, bias, sums);
            t = end;
            if (t == seg.end && t < t1)
                seg.advance(q);
        }
    }
    // the runs of the workgroup together: partial[row block][w][d]
    __shared__ float all[(W + 1) * V][256];
#pragma unroll
    for (int w = 0; w <= W; ++w)
#pragma unroll
        for (int i = 0; i < V; ++i)
            all[w * V + i][threadIdx.x] = sums[w][i];
    __syncthreads();
    const int cols = c.lanes * V;  // channels of the workgroup
    for (int e = threadIdx.x; e < (W + 1) * cols; e += 256) {
        const int w = e / cols, ch = e - w * cols;
        const int dd = col_block * cols + ch;
        if (dd >= a.D)
            continue;
        // (the last lane's vector may have been moved back)
        const int lane = ch / V, back = dd - ch % V + V > a.D && a.D >= V ? dd - ch % V + V - a.D : 0;
        float v = 0.f;
        for (int r = 0; r < c.runs; ++r)
            v += all[w * V + ch % V + back][r * c.lanes + lane];
        a.partial[(block_of * (W + 1) + w) * a.D + dd] = v;
    }
}

// Columns [w][d] of the partial sums to dweight[d][w] and dbias[d].
struct ToTaps {
    float *dweight, *dbias;
    int32_t D, W;
    __device__ __forceinline__ void operator()(int64_t c, float v) const
    {
        const int w = (int)(c / D), d = (int)(c - (int64_t)w * D);
        if (w < W)
            dweight[(int64_t)d * W + w] = v;
        else if (dbias)
            dbias[d] = v;
    }
};

template <typename F> hipError_t by_taps(int32_t W, F &&f)
{
    if (W == 2) return f(std::integral_constant<int, 2>{});
    if (W == 3) return f(std::integral_constant<int, 3>{});
    return f(std::integral_constant<int, 4>{});
}

template <typename T> hipError_t forward(const ConvArgs &a, hipStream_t stream)
{
    const Cut c = forward_cut(a.T, a.D);
    const int64_t states = a.state_out ? (a.B + c.runs - 1) / c.runs : 0;
    // In place, a state may be written only when every run has read it.
    const bool in_place = a.state_out && a.state_out == a.state_in;
    return by_taps(a.W, [&](auto w) {
        auto blocks = [&](int64_t from, int64_t n) {
            return in_launches(n, c.col_blocks, [&](int64_t first, dim3 grid) {
                conv_kernel<decltype(w)::value, T><<<grid, 256, 0, stream>>>(a, c, from + first);
            });
        };
        const hipError_t e = blocks(0, c.row_blocks + (in_place ? 0 : states));
        return e == hipSuccess && in_place ? blocks(c.row_blocks, states) : e;
    });
}
template <typename T> hipError_t step(const ConvArgs &a, hipStream_t stream)
{
    const int64_t threads = a.T * ((a.D + 16 / sizeof(T) - 1) / (16 / sizeof(T)));
    return by_taps(a.W, [&](auto w) {
        return in_launches((threads + 255) / 256, 1, [&](int64_t first, dim3 grid) {
            conv_step_kernel<decltype(w)::value, T><<<grid, 256, 0, stream>>>(a, first);
        });
    });
}
template <typename T> hipError_t backward(const ConvArgs &a, hipStream_t stream)
{
    const Cut c = backward_cut(a.T, a.D);
    const bool empty = a.state_out && (a.offsets || a.T == 0);  // empty sequences are possible
    const int64_t n = c.row_blocks + (empty ? (a.B + c.runs - 1) / c.runs : 0);
    return by_taps(a.W, [&](auto w) {
        return in_launches(n, c.col_blocks, [&](int64_t first, dim3 grid) {
            conv_backward_kernel<decltype(w)::value, T><<<grid, 256, 0, stream>>>(a, c, first);
        });
    });
}

}  // namespace

hipError_t launch_ssm_conv(const ConvArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? forward<bf16_bits>(a, stream) : forward<float>(a, stream);
}

hipError_t launch_ssm_conv_step(const ConvArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? step<bf16_bits>(a, stream) : step<float>(a, stream);
}

int64_t conv_partial_rows(int64_t T, int32_t D) { return backward_cut(T, D).row_blocks; }

hipError_t launch_ssm_conv_backward(const ConvArgs &a, float *dweight, float *dbias, bool bf16,
                                    hipStream_t stream)
{
    const hipError_t e = bf16 ? backward<bf16_bits>(a, stream) : backward<float>(a, stream);
    if (e != hipSuccess)
        return e;
    const int64_t cols = (int64_t)(a.W + 1) * a.D;
    return sum_rows(a.partial, conv_partial_rows(a.T, a.D), cols, cols,
                    ToTaps{dweight, dbias, a.D, a.W}, stream);
}

}  // namespace lbi
