// What the forward scan and its gradient share: the cut of the tokens into
// ranges, the lane layout, the staging of a tile's inputs.
//
// Layout.  A workgroup of four wavefronts holds 64 channels; in a wavefront the
// low four lane bits are the channel and the upper two choose a quarter of the
// N states, NS = ceil(N / 4) of them a lane in registers.  Sums over the states
// are then two exchanges of lane rows for four tokens at a time, B and C are
// read from LDS as broadcasts, and a channel's tokens lie along the walk.
#ifndef LBI_SSM_HPP
#define LBI_SSM_HPP

#include "lbi_block.hpp"

namespace lbi {
namespace {

constexpr int kChannels = 64;   // of a workgroup
constexpr int kPitch = 80;      // floats a row of an LDS plane that lane rows write

// log(1 + e^v) = max(v, 0) + log1p(e), e = e^-|v|.  With w = 1 + e rounded,
// log1p(e) = log(w) + (e - (w - 1)) to first order in what the rounding lost, which
// keeps the relative error at a few 2^-24 where e is small.  NaN gives NaN.
__device__ __forceinline__ float softplus(float v)
{
    const float e = __builtin_amdgcn_exp2f(-fabsf(v) * kLog2e);
    const float w = 1.f + e;
    return fmaf(__builtin_amdgcn_logf(w), kLn2, e - (w - 1.f)) + fmaxf(v, 0.f);
}

// The steps D_t of V channels from delta + delta_bias.  (The choice stands outside
// the loop: V chains of dependent operations at once.)
template <int V> __device__ __forceinline__ void steps_of(bool use_softplus, float (&d)[V])
{
    if (use_softplus) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            d[i] = softplus(d[i]);
    }
}

// The address of a uniform one plus this lane's 32-bit offset.  The offset is made
// opaque at each use: the compiler would otherwise form the sum with the loop's
// invariant part ahead of the loop, two registers for every tensor.
template <typename T> __device__ __forceinline__ T *lane_address(T *uniform, uint32_t bytes)
{
    asm volatile("" : "+v"(bytes));
    return (T *)((char *)uniform + bytes);
}

// A value that is formed here, not where it is used (the compiler would sink sums
// that nothing reads until a walk's end past the walk, and keep their terms).
__device__ __forceinline__ void pin(float &x) { asm volatile("" : "+v"(x)); }

// A token tensor as a staging thread sees it: the rows of a tile begin at a uniform
// address, its own part of them at a 32-bit offset from there (row strides are
// limited to that end).
template <typename T> struct Plane {
    T *base;
    int64_t ld;
    uint32_t offset;  // bytes
    __device__ __forceinline__ Plane(const void *p, int64_t stride, int row, int col)
        : base((T *)p), ld(stride), offset((uint32_t)((row * (int)stride + col) * (int)sizeof(T)))
    {
    }
    __device__ __forceinline__ T *at(int64_t t) const
    {
        return lane_address(base + t * ld, offset);
    }
};
// The same for arrays [.][D][N] of states: `bytes` is the thread's own part.
__device__ __forceinline__ float *part_of(const float *uniform, uint32_t bytes)
{
    return lane_address((float *)uniform, bytes);
}

__device__ __forceinline__ Sequences ssm_sequences(const lbi_ssm_inputs &in)
{
    return {in.offsets, in.T, in.sequences, in.sequences > 0 ? in.T / in.sequences : 0};
}

// The rows t0 .. t1 - 1 of a range.
__device__ __forceinline__ void range_rows(const SsmCut &c, const Sequences &q, int64_t r,
                                           int64_t *t0, int64_t *t1)
{
    if (c.per_sequence > 0) {
        const int64_t s = r / c.per_sequence, end = (s + 1) * q.len;
        *t0 = s * q.len + (r - s * c.per_sequence) * c.tokens;
        *t1 = *t0 + c.tokens < end ? *t0 + c.tokens : end;
    } else {
        *t0 = r * c.tokens;
        *t1 = *t0 + c.tokens < q.T ? *t0 + c.tokens : q.T;
    }
}

// The channels of a workgroup: `left` of them from d0 on, all of group g.
struct Tile {
    int d0, left, group, tile;  // tile: within its group
};
__device__ __forceinline__ Tile tile_of(const lbi_ssm_inputs &in, int index)
{
    const int per_group = in.D / in.G, tiles = (per_group + kChannels - 1) / kChannels;
    Tile t;
    t.group = index / tiles;
    t.tile = index - t.group * tiles;
    const int at = t.tile * kChannels;
    t.d0 = t.group * per_group + at;
    t.left = per_group - at < kChannels ? per_group - at : kChannels;
    return t;
}

// NS states from p on, the first n of them there.
template <int NS> __device__ __forceinline__ void load_states(const float *p, int n, float (&h)[NS])
{
    if constexpr (NS >= 4) {
        Raw<float, NS < 8 ? 4 : 8> r;
        constexpr int V = NS < 8 ? 4 : 8;
#pragma unroll
        for (int i = 0; i < NS; i += V) {
            r.load(p + i, n - i);
#pragma unroll
            for (int j = 0; j < V; ++j)
                h[i + j] = r.v[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < NS; ++i)
            h[i] = i < n ? p[i] : 0.f;
    }
}
template <int NS>
__device__ __forceinline__ void store_states(float *p, int n, const float (&h)[NS])
{
    if (NS >= 4 && n >= NS) {
#pragma unroll
        for (int i = 0; i + 3 < NS; i += 4)
            *(f4_any *)(p + i) = f4{h[i], h[i + 1], h[i + 2], h[i + 3]};
    } else {
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (i < n)
                p[i] = h[i];
    }
}
template <int NS> __device__ __forceinline__ void zero_states(float (&h)[NS])
{
#pragma unroll
    for (int i = 0; i < NS; ++i)
        h[i] = 0.f;
}

// Four tokens' partial sums over a wavefront's four lane rows: lane row g
// returns token g's.
__device__ __forceinline__ float sum_states(const float (&v)[4])
{
    const float even = add_rows<32>(v[0], v[2]);
    const float odd = add_rows<32>(v[1], v[3]);
    return add_rows<16>(even, odd);
}

// The states at the ranges' ends (and, with `heads`, the gradients at their starts),
// each as if its range had been entered with zeros, made whole in place along
// the ranges that follow each other: one thread a channel and state.  A thread has
// the ends of DEEP ranges in flight: its time is that many fewer trips to memory.
template <int DEEP>
__global__ __launch_bounds__(256) void carry_kernel(const SsmArgs a)
{
    const int64_t dN = (int64_t)a.in.D * a.in.N;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= dN)
        return;
    const bool reverse = blockIdx.z == 1;
    const int64_t d = i / a.in.N;
    const int64_t count = a.cut.per_sequence > 0 ? a.cut.per_sequence : a.cut.ranges;
    const int64_t first = (int64_t)blockIdx.y * count;
    const int32_t stops = reverse ? kEnds : kStarts;
    float *ends = reverse ? a.heads : a.ends;
    const float A2 = a.in.A[i] * kLog2e;
    float cur = 0.f;
    for (int64_t k = 0; k < count; k += DEEP) {
        float e[DEEP], w[DEEP];
        int32_t f[DEEP];
#pragma unroll
        for (int j = 0; j < DEEP; ++j) {
            // (past the last range the last one again: nothing is stored then)
            const int64_t at = k + j < count ? k + j : count - 1;
            const int64_t r = first + (reverse ? count - 1 - at : at);
            e[j] = ends[r * dN + i];
            w[j] = a.sums[r * a.in.D + d];
            f[j] = a.flags[r];
        }
#pragma unroll
        for (int j = 0; j < DEEP; ++j) {
            if (k + j < count) {
                const int64_t r = first + (reverse ? count - 1 - (k + j) : k + j);
                cur = f[j] & stops ? e[j] : fmaf(__builtin_amdgcn_exp2f(A2 * w[j]), cur, e[j]);
                ends[r * dN + i] = cur;
            }
        }
    }
}
inline hipError_t launch_carry(const SsmArgs &a, hipStream_t stream)
{
    const int64_t dN = (int64_t)a.in.D * a.in.N;
    const int64_t chains = a.cut.per_sequence > 0 ? a.cut.ranges / a.cut.per_sequence : 1;
    const dim3 grid((unsigned)((dN + 255) / 256), (unsigned)chains, a.heads ? 2 : 1);
    if (a.cut.ranges / chains <= 8)
        carry_kernel<8><<<grid, 256, 0, stream>>>(a);
    else
        carry_kernel<32><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

// Calls f<NS>() for the states a lane holds.
template <typename F> hipError_t by_states(int32_t N, F &&f)
{
    if (N <= 4) return f(std::integral_constant<int, 1>{});
    if (N <= 8) return f(std::integral_constant<int, 2>{});
    if (N <= 16) return f(std::integral_constant<int, 4>{});
    if (N <= 32) return f(std::integral_constant<int, 8>{});
    return f(std::integral_constant<int, 16>{});
}

}  // namespace
}  // namespace lbi

#endif  // LBI_SSM_HPP
