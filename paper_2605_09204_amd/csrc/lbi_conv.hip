// Short causal convolution along packed sequences, channel by channel: forward,
// gradient, and one token a sequence.
//
// A thread owns a few consecutive channels and walks a run of tokens with the
// last W - 1 of them in registers, so every value is loaded once a run (and
// the W - 1 tokens before the run once more, from cache).  The bytes are the
// tensors' own, a few operations for each: the bound is HBM.  Lanes of a
// workgroup lie along the channels (one row's values are contiguous) and, above
// that, along the runs; the length of a run is chosen so that about 2^17
// threads exist, which is what keeps enough loads in flight.
#include "lbi_block.hpp"

namespace lbi {
namespace {

constexpr int64_t kThreads = 1 << 17;  // threads wanted in all
constexpr int kBatch = 4;              // tokens loaded ahead of their use

// How a [tokens][channels] plane is cut: lanes along the channels (a power of
// two), runs beside them in a workgroup of 256, and tokens a run.
struct Cut {
    int lanes, runs, tokens;
    int64_t row_blocks, col_blocks;
};
Cut cut_of(int64_t T, int32_t D, int V, int most_lanes, int least, int most)
{
    const int64_t vec = (D + V - 1) / V;
    int lanes = 1;
    while (lanes < most_lanes && lanes < vec)
        lanes *= 2;
    int tokens = least;
    while (tokens < most && T * vec > (int64_t)tokens * kThreads)
        tokens *= 2;
    const int runs = 256 / lanes;
    const int64_t per = (int64_t)runs * tokens;
    return {lanes, runs, tokens, (T + per - 1) / per, (vec + lanes - 1) / lanes};
}
// Forward: 8 channels a lane, gradient: 4 (its sums and its tokens in flight
// take twice the registers).
Cut forward_cut(int64_t T, int32_t D) { return cut_of(T, D, 8, 32, 4, 64); }
Cut backward_cut(int64_t T, int32_t D) { return cut_of(T, D, 4, 64, 8, 256); }

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

// The W - 1 tokens before row t of a sequence, oldest first: rows of x, or of
// the state where the sequence has not that many.
template <int W, int V, typename T>
__device__ __forceinline__ void load_window(const ConvArgs &a, const Segment &seg, int64_t t, int d,
                                            int left, float (&win)[W - 1][V])
{
    const int64_t slot = a.state_in ? state_row(a.slots, a.n_slots, seg.seq) : -1;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int64_t row = t - (W - 1) + j;
        if (row >= seg.start) {
            load_some<V>((const T *)a.x + row * a.ld_x + d, left, win[j]);
        } else if (slot >= 0) {
            const int64_t k = (W - 1) + (row - seg.start);
            load_some<V>((const T *)a.state_in + (slot * (W - 1) + k) * a.D + d, left, win[j]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                win[j][i] = 0.f;
        }
    }
}

// The state after sequence s: the last W - 1 of its old state and its tokens.
template <int W, typename T>
__device__ __forceinline__ void write_state(const ConvArgs &a, const Sequences &q, int64_t s, int d,
                                            int left)
{
    const int64_t slot = state_row(a.slots, a.n_slots, s);
    if (slot < 0)
        return;
    const int64_t start = q.at(s), len = q.at(s + 1) - start;
    float v[W - 1][8];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int64_t p = len - (W - 1) + j;
        if (p >= 0)
            load_some<8>((const T *)a.x + (start + p) * a.ld_x + d, left, v[j]);
        else if (a.state_in && len >= 0)
            load_some<8>((const T *)a.state_in + (slot * (W - 1) + len + j) * a.D + d, left, v[j]);
        else
            load_some<8>((const T *)a.x, 0, v[j]);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        store_some<8>((T *)a.state_out + (slot * (W - 1) + j) * a.D + d, left, v[j]);
}

// Workgroups first .. first + row_blocks - 1 convolve, those from row_blocks on
// write states.
template <int W, typename T>
__global__ __launch_bounds__(256) void conv_kernel(const ConvArgs a, const Cut c, int64_t first)
{
    constexpr int V = 8;
    const Sequences q = {a.offsets, a.T, a.B, a.B > 0 ? a.T / a.B : 0};
    const int d = ((int)blockIdx.y * c.lanes + threadIdx.x % c.lanes) * V, left = a.D - d;
    if (left <= 0)
        return;
    const int64_t block = first + blockIdx.x;
    const int64_t run = block * c.runs + threadIdx.x / c.lanes;
    if (block >= c.row_blocks) {
        const int64_t s = run - c.row_blocks * c.runs;
        if (s < a.B)
            write_state<W, T>(a, q, s, d, left);
        return;
    }
    const int64_t t0 = run * c.tokens, t1 = t0 + c.tokens < a.T ? t0 + c.tokens : a.T;
    if (t0 >= t1)
        return;
    const T *x = (const T *)a.x + d;
    T *out = (T *)a.out + d;
    float k[W][V], bias[V], win[W - 1][V];
    Raw<T, V> next[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
        next[b].load(x + (t0 + b) * a.ld_x, t0 + b < t1 ? left : 0);
    load_taps<W, V>(a.weight, d, left, k);
    load_some<V>(a.bias ? a.bias + d : a.bias, a.bias ? left : 0, bias);
    Segment seg;
    seg.enter(q, t0);
    load_window<W, V, T>(a, seg, t0, d, left, win);
    for (int64_t t = t0; t < t1; t += kBatch) {
        float cur[kBatch][V];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            next[b].unpack(cur[b]);
            next[b].load(x + (t + kBatch + b) * a.ld_x, t + kBatch + b < t1 ? left : 0);
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (t + b >= t1)
                break;
            if (t + b == seg.end) {
                seg.advance(q);
                load_window<W, V, T>(a, seg, t + b, d, left, win);
            }
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float v = bias[i];
#pragma unroll
                for (int w = 0; w < W - 1; ++w)
                    v += k[w][i] * win[w][i];
                v += k[W - 1][i] * cur[b][i];
                y[i] = a.silu ? silu(v) : v;
#pragma unroll
                for (int w = 0; w < W - 2; ++w)
                    win[w][i] = win[w + 1][i];
                win[W - 2][i] = cur[b][i];
            }
            store_some<V>(out + (t + b) * a.ld_out, left, y);
        }
    }
}

template <int W, typename T>
__global__ __launch_bounds__(256) void conv_step_kernel(const ConvArgs a)
{
    constexpr int V = 8;
    const int64_t vec = (a.D + V - 1) / V;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
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

// Gradient.  Walking forward, token t adds dv_t weight_{W-1-j} to the gradient
// of token t - j, j = 0 .. W - 1, so that of token t - (W - 1) is then whole.  A
// run walks up to W - 1 tokens past its end to complete its own; the run that
// holds a sequence's first token completes the gradient of its old state.
template <int W, typename T>
__global__ __launch_bounds__(256) void conv_backward_kernel(const ConvArgs a, const Cut c)
{
    constexpr int V = 4;
    const Sequences q = {a.offsets, a.T, a.B, a.B > 0 ? a.T / a.B : 0};
    const int d = ((int)blockIdx.y * c.lanes + threadIdx.x % c.lanes) * V, left = a.D - d;
    const int64_t run = (int64_t)blockIdx.x * c.runs + threadIdx.x / c.lanes;
    if ((int64_t)blockIdx.x >= c.row_blocks) {
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
    const int64_t t0 = run * c.tokens, t1 = t0 + c.tokens < a.T ? t0 + c.tokens : a.T;
    float sums[W + 1][V];  // dweight, dbias
#pragma unroll
    for (int w = 0; w <= W; ++w)
#pragma unroll
        for (int i = 0; i < V; ++i)
            sums[w][i] = 0.f;
    if (left > 0 && t0 < t1) {
        const T *x = (const T *)a.x + d, *dy = (const T *)a.dout + d;
        T *dx = (T *)a.out + d;
        float k[W][V], bias[V], win[W - 1][V], wait[W - 1][V];
        Raw<T, V> nx[kBatch], ny[kBatch];
        const int64_t last = t1 + W - 1 < a.T ? t1 + W - 1 : a.T;  // rows that may be walked
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int n = t0 + b < last ? left : 0;
            nx[b].load(x + (t0 + b) * a.ld_x, n);
            ny[b].load(dy + (t0 + b) * a.ld_dout, n);
        }
        load_taps<W, V>(a.weight, d, left, k);
        load_some<V>(a.bias ? a.bias + d : a.bias, a.bias ? left : 0, bias);
        Segment seg;
        seg.enter(q, t0);
        load_window<W, V, T>(a, seg, t0, d, left, win);
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i)
                wait[j][i] = 0.f;
        bool done = false;
        for (int64_t tb = t0; !done; tb += kBatch) {
            float cx[kBatch][V], cy[kBatch][V];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                nx[b].unpack(cx[b]);
                ny[b].unpack(cy[b]);
                const int64_t t = tb + kBatch + b;
                const int n = t < last ? left : 0;
                nx[b].load(x + t * a.ld_x, n);
                ny[b].load(dy + t * a.ld_dout, n);
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int64_t t = tb + b;
                if (done)
                    break;
                if (t == seg.end) {  // t < t1 here: else the walk has ended
                    seg.advance(q);
                    load_window<W, V, T>(a, seg, t, d, left, win);
#pragma unroll
                    for (int j = 0; j < W - 1; ++j)
#pragma unroll
                        for (int i = 0; i < V; ++i)
                            wait[j][i] = 0.f;
                }
                const bool own = t < t1;
                float whole[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float v = bias[i];
#pragma unroll
                    for (int w = 0; w < W - 1; ++w)
                        v += k[w][i] * win[w][i];
                    v += k[W - 1][i] * cx[b][i];
                    float g = cy[b][i];
                    if (a.silu)
                        g *= silu_slope(v, sigmoid(v));
                    const float mine = own ? g : 0.f;
#pragma unroll
                    for (int w = 0; w < W - 1; ++w)
                        sums[w][i] += mine * win[w][i];
                    sums[W - 1][i] += mine * cx[b][i];
                    sums[W][i] += mine;
                    whole[i] = wait[W - 2][i] + g * k[0][i];
#pragma unroll
                    for (int j = W - 2; j > 0; --j)
                        wait[j][i] = wait[j - 1][i] + g * k[W - 1 - j][i];
                    wait[0][i] = g * k[W - 1][i];
#pragma unroll
                    for (int w = 0; w < W - 2; ++w)
                        win[w][i] = win[w + 1][i];
                    win[W - 2][i] = cx[b][i];
                }
                const bool starts = seg.start >= t0 && seg.start < t1;  // the sequence starts here
                const int64_t row = t - (W - 1);
                if (row >= seg.start) {
                    if (row >= t0)
                        store_some<V>(dx + row * a.ld_out, left, whole);
                } else if (starts && a.state_out) {
                    const int64_t j = (W - 1) + (row - seg.start);
                    store_some<V>((T *)a.state_out + (seg.seq * (W - 1) + j) * a.D + d, left, whole);
                }
                if (t + 1 == seg.end) {
                    // wait[j] belongs to row t - j, that is to row W - 2 - j of state_out
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) {
                        float v[V];
                        const int64_t from = (seg.seq * (W - 1) + (W - 2 - j)) * a.D + d;
                        load_some<V>((const T *)a.dstate_out + (a.dstate_out ? from : 0),
                                     a.dstate_out ? left : 0, v);
#pragma unroll
                        for (int i = 0; i < V; ++i)
                            v[i] += wait[j][i];
                        const int64_t r = t - j;
                        if (r >= seg.start) {
                            if (r >= t0 && r < t1)
                                store_some<V>(dx + r * a.ld_out, left, v);
                        } else if (starts && a.state_out) {
                            const int64_t m = (W - 1) + (r - seg.start);
                            store_some<V>((T *)a.state_out + (seg.seq * (W - 1) + m) * a.D + d,
                                          left, v);
                        }
                    }
                    done = t + 1 >= t1;
                } else {
                    done = t + 1 >= last;
                }
            }
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
        const int dd = (int)blockIdx.y * cols + ch;
        if (dd >= a.D)
            continue;
        float v = 0.f;
        for (int r = 0; r < c.runs; ++r)
            v += all[w * V + ch % V][r * c.lanes + ch / V];
        a.partial[((int64_t)blockIdx.x * (W + 1) + w) * a.D + dd] = v;
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
        const int64_t n = c.row_blocks + (in_place ? 0 : states);
        if (n > 0)
            conv_kernel<decltype(w)::value, T>
                <<<dim3((unsigned)n, (unsigned)c.col_blocks), 256, 0, stream>>>(a, c, 0);
        if (in_place && states > 0)
            conv_kernel<decltype(w)::value, T>
                <<<dim3((unsigned)states, (unsigned)c.col_blocks), 256, 0, stream>>>(a, c,
                                                                                     c.row_blocks);
        return hipGetLastError();
    });
}
template <typename T> hipError_t step(const ConvArgs &a, hipStream_t stream)
{
    const int64_t threads = a.T * ((a.D + 7) / 8);
    return by_taps(a.W, [&](auto w) {
        conv_step_kernel<decltype(w)::value, T>
            <<<dim3((unsigned)((threads + 255) / 256)), 256, 0, stream>>>(a);
        return hipGetLastError();
    });
}
template <typename T> hipError_t backward(const ConvArgs &a, hipStream_t stream)
{
    const Cut c = backward_cut(a.T, a.D);
    const bool empty = a.state_out && (a.offsets || a.T == 0);  // empty sequences are possible
    const int64_t n = c.row_blocks + (empty ? (a.B + c.runs - 1) / c.runs : 0);
    return by_taps(a.W, [&](auto w) {
        if (n > 0)
            conv_backward_kernel<decltype(w)::value, T>
                <<<dim3((unsigned)n, (unsigned)c.col_blocks), 256, 0, stream>>>(a, c);
        return hipGetLastError();
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
