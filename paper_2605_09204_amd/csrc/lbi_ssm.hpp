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

// A2 = A log2(e), kept finite: rows past a tile's last one have D_t = 0, and 0 (-inf) is NaN.
__device__ __forceinline__ float power_rate(float A)
{
    const float A2 = A * kLog2e;
    return A2 < -3.4e38f ? -3.4e38f : A2;
}
// A token's decay exp(D_t A) = 2^p, p = D_t A2.  The hardware's 2^p
// is a little low on average where it matters, close below 1: by 0.11 units of the
// last place for p in (-0.001, 0) and 0.07 in (-0.01, -0.001), and products of hundreds of
// such decays carry that on (the gradient of A over 4600 tokens: 4e-6 off).  6e-9 added to p
// brings these to 0.04 and 0.00; 2^0 stays 1.
__device__ __forceinline__ float decay(float step, float A2)
{
    return __builtin_amdgcn_exp2f(fmaf(step, A2, 6e-9f));
}

// h 2^p, p = whole + part: the product over a range's decays (p = A2 sum D_t), also where 2^p alone
// passes float32's range and h 2^p does not (A > 0, and h zero or small).
__device__ __forceinline__ float power_parts(float p, int *whole)
{
    p = fminf(fmaxf(p, -1e5f), 1e5f);
    const float w = rintf(p);
    *whole = (int)w;
    return __builtin_amdgcn_exp2f(p - w);
}
__device__ __forceinline__ float grown(float h, float part, int whole)
{
    return __builtin_amdgcn_ldexpf(h * part, whole);
}
__device__ __forceinline__ float grown(float h, float p)
{
    int whole;
    const float part = power_parts(p, &whole);
    return grown(h, part, whole);
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

// The kernel's own arguments, read again from where they were passed: within a loop
// over tiles, so that some fifty pointers and strides are not held in scalar
// registers (of which there are 102; the compiler spilled them to lanes of vector
// registers, and an eighth of the gradient kernel's instructions fetched them back).
typedef const __attribute__((address_space(4))) SsmArgs *PassedArgs;
__device__ __forceinline__ PassedArgs passed()
{
    PassedArgs p = (PassedArgs)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return p;
}

// A staging thread's part of a tile's rows in a token tensor, as a 32-bit offset
// from the uniform address of the first row (row strides are limited to that end).
template <typename T> struct Plane {
    uint32_t offset;  // bytes
    __device__ __forceinline__ Plane(int64_t ld, int row, int col)
        : offset((uint32_t)((row * (int)ld + col) * (int)sizeof(T)))
    {
    }
    __device__ __forceinline__ T *at(const void *base, int64_t ld, int64_t t) const
    {
        return lane_address((T *)base + t * ld, offset);
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
// V values of LDS, at an address aligned to them (16 bytes at most).
template <int V> __device__ __forceinline__ void read_lds(const float *p, float (&v)[V])
{
    if constexpr (V == 2) {
        const f2 q = *(const f2 *)p;
        v[0] = q.x; v[1] = q.y;
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const f4 q = *(const f4 *)(p + i);
            v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
        }
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
// the ranges that follow each other: one lane a channel and state.  Its time is trips to
// memory, so each of WAVES wavefronts has the ends of DEEP consecutive ranges in flight;
// the wavefronts exchange what their ranges do to a state that enters them (the end from zero, and
// the power of two that decays it), and each then walks its ranges again from the state that does enter.
// The ranges of 32768 tokens, 12288 states: 9.6 us (with decays as plain factors, which overflow
// where a channel grows, 7.4; so by one wavefront in batches of 32 ranges 15.4).
// Up to 8 ranges one trip does, with one wavefront (5.6 us for 8 sequences of 24576 states).
template <int DEEP, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void carry_kernel(const SsmArgs a)
{
    struct Map {
        float end, power;  // power NaN: a sequence starts within, and what enters is dropped
    };
    __shared__ Map maps[WAVES > 1 ? 2 : 1][WAVES > 1 ? WAVES : 1][64];
    const int lane = threadIdx.x % 64, wave = (int)uniform(threadIdx.x / 64);
    const int64_t dN = (int64_t)a.in.D * a.in.N;
    int64_t i = (int64_t)blockIdx.x * 64 + lane;
    const bool live = i < dN;
    if (!live)
        i = dN - 1;  // such lanes only help with the flags
    const bool reverse = blockIdx.z == 1;
    const int64_t d = i / a.in.N;
    const int64_t count = a.cut.per_sequence > 0 ? a.cut.per_sequence : a.cut.ranges;
    const int64_t first = (int64_t)blockIdx.y * count;
    const int32_t stops = reverse ? kEnds : kStarts;
    const float A2 = power_rate(a.in.A[i]);
    const int64_t from = reverse ? first + count - 1 : first, one = reverse ? -1 : 1;
    const int64_t down = one * dN, along = one * a.in.D;  // to the next range
    float cur = 0.f;
    int parity = 0;
    for (int64_t k = 0; k < count; k += DEEP * WAVES) {
        const int64_t k0 = k + wave * DEEP;
        const int mine = k0 >= count ? 0 : (count - k0 < DEEP ? (int)(count - k0) : DEEP);
        const int64_t at = from + one * (mine > 0 ? k0 : k);  // a range that is there
        float *ends = (reverse ? a.heads : a.ends) + at * dN + i;
        const float *sums = a.sums + at * a.in.D + d;
        const uint64_t stop =
            __ballot(lane < mine && (a.flags[at + (lane < mine ? lane * one : 0)] & stops));
        float e[DEEP], w[DEEP];  // ends; powers, then their parts
        int n[DEEP];
        {
            const float *p = ends, *s = sums;
#pragma unroll
            for (int j = 0; j < DEEP; ++j) {
                e[j] = *p;
                w[j] = *s;
                p += j + 1 < mine ? down : 0;
                s += j + 1 < mine ? along : 0;
            }
        }
        float power = 0.f;  // of all of them
#pragma unroll
        for (int j = 0; j < DEEP; ++j) {
            const float p = A2 * w[j];
            power += j < mine ? p : 0.f;
            w[j] = power_parts(p, &n[j]);
        }
        if constexpr (WAVES > 1) {
            Map m = {0.f, stop ? __builtin_nanf("") : power};
#pragma unroll
            for (int j = 0; j < DEEP; ++j) {
                if (j < mine) {
                    const bool drop = stop >> j & 1;
                    m.end = drop ? e[j] : e[j] + grown(m.end, w[j], n[j]);
                }
            }
            maps[parity][wave][lane] = m;
            __syncthreads();
            float enters = cur;
#pragma unroll
            for (int v = 0; v < WAVES; ++v) {
                const Map o = maps[parity][v][lane];
                if (v == wave)
                    enters = cur;
                cur = o.power != o.power ? o.end : o.end + grown(cur, o.power);
            }
            parity ^= 1;  // the next maps go where nobody reads any more
#pragma unroll
            for (int j = 0; j < DEEP; ++j) {
                if (j < mine) {
                    enters = stop >> j & 1 ? e[j] : e[j] + grown(enters, w[j], n[j]);
                    if (live)
                        *ends = enters;
                    ends += down;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < DEEP; ++j) {
                if (j < mine) {
                    cur = stop >> j & 1 ? e[j] : e[j] + grown(cur, w[j], n[j]);
                    if (live)
                        *ends = cur;
                    ends += down;
                }
            }
        }
    }
}
inline hipError_t launch_carry(const SsmArgs &a, hipStream_t stream)
{
    const int64_t dN = (int64_t)a.in.D * a.in.N;
    const int64_t chains = a.cut.per_sequence > 0 ? a.cut.ranges / a.cut.per_sequence : 1;
    const int64_t count = a.cut.ranges / chains;
    const dim3 grid((unsigned)((dN + 63) / 64), (unsigned)chains, a.heads ? 2 : 1);
    if (count <= 8)
        carry_kernel<8, 1><<<grid, 64, 0, stream>>>(a);
    else if (count <= 32)
        carry_kernel<8, 4><<<grid, 256, 0, stream>>>(a);
    else
        carry_kernel<32, 4><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

// launch(arguments, workgroups) for all ranges.
template <typename F> hipError_t over_ranges(const SsmArgs &a, F &&launch)
{
    return in_launches(a.cut.ranges, a.cut.tiles, [&](int64_t first, dim3 grid) {
        SsmArgs b = a;
        b.cut.first = (uint32_t)first;
        launch(b, grid);
    });
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
