// What the norms' kernels share: rows in registers, eight consecutive features a
// lane and vector, sums over a row's lanes, and how many lanes a row gets.
#ifndef LBI_NORM_ROWS_HPP
#define LBI_NORM_ROWS_HPP

#include "lbi_block.hpp"

namespace lbi {
namespace {

// Sums v[] over the LANES lanes of a row; red: 2 x 16 floats of LDS per value.
template <int LANES, int NVAL> __device__ __forceinline__ void row_sum(float (&v)[NVAL], float *red,
                                                                       int parity)
{
#pragma unroll
    for (int i = 0; i < NVAL; ++i)
        v[i] = lanes_sum<(LANES < 64 ? LANES : 64)>(v[i]);
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64;
        float *r = red + parity * NVAL * W;  // the other half may still be read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < NVAL; ++i)
                r[i * W + (threadIdx.x >> 6)] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NVAL; ++i) {
            v[i] = r[i * W];
#pragma unroll
            for (int w = 1; w < W; ++w)
                v[i] += r[i * W + w];
        }
    }
}

// s = x + residual of a row (x alone without one), written to residual_out where that is.
template <typename X, typename R, int NV>
__device__ __forceinline__ void load_sum(const NormArgs &a, int64_t row, const int (&col)[NV],
                                         const int (&left)[NV], float (&s)[NV][8])
{
    const X *x = (const X *)a.x + row * a.ld_x;
#pragma unroll
    for (int j = 0; j < NV; ++j)
        load_some<8>(x + col[j], left[j], s[j]);
    if (a.residual) {
        const R *r = (const R *)a.residual + row * a.ld_residual;
        float t[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j)
            load_some<8>(r + col[j], left[j], t[j]);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s[j][i] += t[j][i];
        if (a.residual_out) {
            R *o = (R *)a.residual_out + row * a.ld_residual_out;
#pragma unroll
            for (int j = 0; j < NV; ++j)
                store_some<8>(o + col[j], left[j], s[j]);
        }
    }
}

constexpr int64_t kBlocks = 2048;          // forward: 8 workgroups a CU
constexpr int64_t kBackwardBlocks = 1024;  // also the rows of partial sums

struct Shape {
    int lanes, nv, rows;  // lanes of a row, vectors a lane, rows a workgroup
};
// Up to 1024 features a wavefront takes a row, above that a workgroup: measured in bf16
// at 64 to 16384 rows, a workgroup instead costs rows of 1024 features 3 to 26 per cent forward
// and up to 61 in the gradient, and a wavefront instead costs rows of 2048 up to 24 forward.  From
// 4097 to 8192 features 1024 lanes instead of 256 change the forward by 0 to 5 per cent either
// way and the gradient (bf16) from 39.6 to 33.7 us at 3000 rows of 4100, from 21.3 to 23.7 at 1500 of 8192.
Shape shape_of(int32_t D)
{
    const int vec = (D + 7) / 8;
    if (vec <= 16) return {16, 1, 16};
    if (vec <= 64) return {64, 1, 4};
    if (vec <= 128) return {64, 2, 4};
    if (vec <= 256) return {256, 1, 1};
    if (vec <= 512) return {256, 2, 1};
    if (vec <= 1024) return {256, 4, 1};
    return {1024, 2, 1};
}

// Calls f<LANES, NV>() for the shape.
template <typename F> hipError_t by_shape(const Shape &s, F &&f)
{
    if (s.lanes == 16) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    if (s.lanes == 64) {
        if (s.nv == 1) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
        return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
    }
    if (s.lanes == 256) {
        if (s.nv == 1) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
        if (s.nv == 2) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
        return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 4>{});
    }
    return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
}
int64_t block_count(int64_t T, int rows, int64_t most)
{
    const int64_t n = (T + rows - 1) / rows;
    return n < most ? n : most;
}

struct ToVector {
    float *out;
    __device__ __forceinline__ void operator()(int64_t c, float v) const { out[c] = v; }
};

}  // namespace
}  // namespace lbi

#endif  // LBI_NORM_ROWS_HPP
