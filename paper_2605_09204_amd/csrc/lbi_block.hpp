// Device helpers shared by the kernels of the region block's operators
// (include/lbi_block.h): eight token values at a time in float32 registers,
// sums over a wavefront, packed sequences.
#ifndef LBI_BLOCK_HPP
#define LBI_BLOCK_HPP

#include "lbi_block_internal.h"
#include "lbi_device.hpp"

namespace lbi {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.69314718055994531f;

// Token rows start at any element: global loads and stores of 16 and 8 bytes
// need no alignment on gfx950 beyond the element's.
typedef u4 u4_any __attribute__((aligned(2)));
typedef u2 u2_any __attribute__((aligned(2)));
typedef uint32_t u1_any __attribute__((aligned(2)));
typedef f4 f4_any __attribute__((aligned(4)));

// Storage types: float, and bf16 as its 16 bits.
typedef uint16_t bf16_bits;

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(bf16_bits x) { return bitsf((uint32_t)x << 16); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16_bits narrow<bf16_bits>(float x)
{
    return __builtin_bit_cast(bf16_bits, (__bf16)x);
}
__device__ __forceinline__ uint32_t narrow_pair(float x0, float x1)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{x0, x1}, bf16x2));
}

// V consecutive values of a token row as they are stored (V = 2, 4 or 8): loads
// that stay in flight until unpack().  Only the first n values are there (n may
// be 0 or less, or V and more): the others read as zero and are not written.
template <typename T, int V> struct Raw;
template <int V> struct Raw<float, V> {
    float v[V];
    __device__ __forceinline__ void load(const float *p, int n)
    {
        if (n >= V) {
            if constexpr (V == 2) {
                const u2 q = *(const u2_any *)p;
                v[0] = bitsf(q.x); v[1] = bitsf(q.y);
            } else {
#pragma unroll
                for (int i = 0; i < V; i += 4) {
                    const f4 q = *(const f4_any *)(p + i);
                    v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                v[i] = i < n ? p[i] : 0.f;
        }
    }
    __device__ __forceinline__ void unpack(float (&x)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V; ++i)
            x[i] = v[i];
    }
};
template <int V> struct Raw<bf16_bits, V> {
    uint32_t w[V / 2];
    __device__ __forceinline__ void load(const bf16_bits *p, int n)
    {
        if (n >= V) {
            if constexpr (V == 8) {
                const u4 q = *(const u4_any *)p;
                w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
            } else if constexpr (V == 4) {
                const u2 q = *(const u2_any *)p;
                w[0] = q.x; w[1] = q.y;
            } else {
                w[0] = *(const u1_any *)p;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i)
                w[i] = (2 * i < n ? (uint32_t)p[2 * i] : 0u) |
                       (2 * i + 1 < n ? (uint32_t)p[2 * i + 1] << 16 : 0u);
        }
    }
    __device__ __forceinline__ void unpack(float (&x)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            x[2 * i] = bitsf(w[i] << 16);
            x[2 * i + 1] = bitsf(w[i] & kHighHalf);
        }
    }
};
template <int V, typename T>
__device__ __forceinline__ void load_some(const T *p, int n, float (&v)[V])
{
    Raw<T, V> r;
    r.load(p, n);
    r.unpack(v);
}
template <int V> __device__ __forceinline__ void store_all(float *p, const float (&v)[V])
{
    if constexpr (V == 2) {
        *(u2_any *)p = u2{fbits(v[0]), fbits(v[1])};
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4)
            *(f4_any *)(p + i) = f4{v[i], v[i + 1], v[i + 2], v[i + 3]};
    }
}
template <int V> __device__ __forceinline__ void store_all(bf16_bits *p, const float (&v)[V])
{
    if constexpr (V == 8)
        *(u4_any *)p = u4{narrow_pair(v[0], v[1]), narrow_pair(v[2], v[3]),
                          narrow_pair(v[4], v[5]), narrow_pair(v[6], v[7])};
    else if constexpr (V == 4)
        *(u2_any *)p = u2{narrow_pair(v[0], v[1]), narrow_pair(v[2], v[3])};
    else
        *(u1_any *)p = narrow_pair(v[0], v[1]);
}
template <int V, typename T>
__device__ __forceinline__ void store_some(T *p, int n, const float (&v)[V])
{
    if (n >= V) {
        store_all<V>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n)
                p[i] = narrow<T>(v[i]);
    }
}

// Lane exchanges across the four 16-lane rows of a wavefront: (a, b) become
// (a's even rows and b's even rows, a's odd rows and b's odd rows) for ROW 16,
// the same with the wavefront's halves for ROW 32.
template <int ROW> __device__ __forceinline__ void swap_rows(float &a, float &b)
{
    if constexpr (ROW == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(fbits(a), fbits(b), false, false);
        a = bitsf(r[0]);
        b = bitsf(r[1]);
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(fbits(a), fbits(b), false, false);
        a = bitsf(r[0]);
        b = bitsf(r[1]);
    }
}
template <int ROW> __device__ __forceinline__ float add_rows(float a, float b)
{
    swap_rows<ROW>(a, b);
    return a + b;
}

// The sum, or the largest bit pattern, over an aligned group of N lanes
// (N = 4 .. 64), in every lane of the group.
template <int N> __device__ __forceinline__ float lanes_sum(float x)
{
    x += xchg<1>(x);
    x += xchg<2>(x);
    if constexpr (N >= 8) x += xchg<7>(x);
    if constexpr (N >= 16) x += xchg<8>(x);
    if constexpr (N >= 32) x = add_rows<16>(x, x);
    if constexpr (N >= 64) x = add_rows<32>(x, x);
    return x;
}
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
template <int N> __device__ __forceinline__ uint32_t lanes_max(uint32_t x)
{
    x = umax(x, fbits(xchg<1>(bitsf(x))));
    x = umax(x, fbits(xchg<2>(bitsf(x))));
    if constexpr (N >= 8) x = umax(x, fbits(xchg<7>(bitsf(x))));
    if constexpr (N >= 16) x = umax(x, fbits(xchg<8>(bitsf(x))));
    if constexpr (N >= 32) {
        float a = bitsf(x), b = a;
        swap_rows<16>(a, b);
        x = umax(fbits(a), fbits(b));
    }
    if constexpr (N >= 64) {
        float a = bitsf(x), b = a;
        swap_rows<32>(a, b);
        x = umax(fbits(a), fbits(b));
    }
    return x;
}

// The address of a uniform one plus this lane's 32-bit offset.  The offset is made
// opaque at each use: the compiler would otherwise form the sum with the loop's
// invariant part ahead of the loop, two registers for every tensor.
template <typename T> __device__ __forceinline__ T *lane_address(T *uniform, uint32_t bytes)
{
    asm volatile("" : "+v"(bytes));
    return (T *)((char *)uniform + bytes);
}

// A value that all lanes of the wavefront have, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)x) |
           (int64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32;
}

// A value that is formed here, not where it is used (the compiler would sink sums
// that nothing reads until a walk's end past the walk, and keep their terms).
__device__ __forceinline__ void pin(float &x) { asm volatile("" : "+v"(x)); }

// 1 / (1 + e^-x); 0 and 1 at the ends of the range, NaN for NaN.  The exponent's rounding makes the
// relative error about |x| 1e-7 far below zero, where the value itself is e^x.
__device__ __forceinline__ float sigmoid(float x)
{
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-x * kLog2e));
}
__device__ __forceinline__ float silu(float x) { return x * sigmoid(x); }
// d silu / dx, given g = sigmoid(x).
__device__ __forceinline__ float silu_slope(float x, float g) { return g * (1.f + x * (1.f - g)); }

// Packed sequences.  Everything that a kernel takes from `offsets` passes
// through these, which keep rows within 0 .. T whatever the array holds.
struct Sequences {
    const int64_t *offsets;  // NULL: `len` rows each
    int64_t T, B, len;

    __device__ __forceinline__ int64_t at(int64_t i) const
    {
        if (!offsets)
            return i * len;
        const int64_t o = offsets[i];
        return o < 0 ? 0 : (o > T ? T : o);
    }
    // The sequence that holds row t (0 <= t < T): the last one that starts at
    // or before it, so never an empty one that starts there as well.
    __device__ __forceinline__ int64_t find(int64_t t) const
    {
        if (!offsets)
            return len > 0 ? t / len : 0;
        int64_t lo = 0, hi = B;  // at(lo) <= t < at(hi)
        while (hi - lo > 1) {
            const int64_t mid = (lo + hi) >> 1;
            if (at(mid) <= t) lo = mid;
            else hi = mid;
        }
        return lo;
    }
    // The same by a whole wavefront with one t: 64 offsets at a time, so one or two
    // trips to memory instead of one a halving.
    __device__ __forceinline__ int64_t find_together(int64_t t) const
    {
        if (!offsets)
            return len > 0 ? t / len : 0;
        const int lane = threadIdx.x & 63;
        int64_t lo = 0, n = B;  // among lo .. lo + n - 1
        while (n > 1) {
            const int64_t step = (n + 63) / 64, i = lo + lane * step;
            const int before = __popcll(__ballot(lane * step < n && at(i) <= t));
            const int64_t skip = before > 0 ? (before - 1) * step : 0;
            lo += skip;
            n = n - skip < step ? n - skip : step;
        }
        return lo;
    }
    // The next sequence after i that is not empty, or B.
    __device__ __forceinline__ int64_t next(int64_t i) const
    {
        for (++i; i < B && at(i + 1) <= at(i); ++i) {}
        return i;
    }
};

// A walk along the packed rows: the sequence of row t and its rows
// start .. end - 1, always with start <= t < end <= T.
struct Segment {
    int64_t seq, start, end;

    // together: by all lanes of a wavefront, with the same t
    __device__ __forceinline__ void enter(const Sequences &q, int64_t t, bool together)
    {
        seq = together ? q.find_together(t) : q.find(t);
        start = q.at(seq);
        end = q.at(seq + 1);
        if (start > t) start = t;  // only with offsets that do not ascend
        if (end <= t) end = q.T;
    }
    // To the sequence that starts at row t = end (t < T).
    __device__ __forceinline__ void advance(const Sequences &q)
    {
        const int64_t t = end, n = q.next(seq);
        seq = n < q.B ? n : q.B - 1;
        start = t;
        end = q.at(seq + 1);
        if (end <= t) end = q.T;
    }
};

// The row of a state tensor that sequence i uses, or -1.
__device__ __forceinline__ int64_t state_row(const int32_t *slots, int32_t n_slots, int64_t i)
{
    if (!slots)
        return i;
    const int32_t s = slots[i];
    return s >= 0 && s < n_slots ? s : -1;
}

// Rows of `cols` workgroups of 256 in as many launches as they need: launch(first row, workgroups).
template <typename F> hipError_t in_launches(int64_t rows, int64_t cols, F &&launch)
{
    const int64_t per = kMostGroups / cols;
    for (int64_t first = 0; first < rows; first += per) {
        const int64_t n = rows - first < per ? rows - first : per;
        launch(first, dim3((unsigned)(n * cols)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

// store(c, the sum over r < rows of partial[r * pitch + c]) for c < cols, in a
// fixed order.  16 row groups x 64 columns a workgroup, so that a few hundred
// rows are a few dozen loads deep.
constexpr int kSumGroups = 16;
template <typename Store>
__global__ __launch_bounds__(64 * kSumGroups) void sum_rows_kernel(const float *partial,
                                                                   int64_t rows, int64_t pitch,
                                                                   int64_t cols, Store store)
{
    __shared__ float sums[kSumGroups][64];
    const int lane = threadIdx.x & 63, group = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float v = 0.f;
    if (c < cols) {
        const float *p = partial + c;
        int64_t r = group;
        for (; r + 7 * kSumGroups < rows; r += 8 * kSumGroups) {
            float t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                t[i] = p[(r + i * kSumGroups) * pitch];
            v += ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
        }
        for (; r < rows; r += kSumGroups)
            v += p[r * pitch];
    }
    sums[group][lane] = v;
    __syncthreads();
    if (group == 0 && c < cols) {
#pragma unroll
        for (int g = 1; g < kSumGroups; ++g)
            v += sums[g][lane];
        store(c, v);
    }
}
template <typename Store>
hipError_t sum_rows(const float *partial, int64_t rows, int64_t pitch, int64_t cols, Store store,
                    hipStream_t stream)
{
    sum_rows_kernel<<<dim3((unsigned)((cols + 63) / 64)), dim3(64 * kSumGroups), 0, stream>>>(
        partial, rows, pitch, cols, store);
    return hipGetLastError();
}

}  // namespace
}  // namespace lbi

#endif  // LBI_BLOCK_HPP
