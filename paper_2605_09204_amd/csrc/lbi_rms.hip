// Root-mean-square norm with the residual's addition: forward in the token type
// or in 8 bits with scales, and its gradient.
//
// A row is read once and stays in registers as float32, eight consecutive
// features a lane and vector; its sum of squares (and, for scales, its largest
// magnitudes; for the gradient, its dot product with g) is formed over the
// lanes of the row, then the row is written.  So each form moves exactly the
// bytes it has to, and the bound is HBM.  A group of LANES lanes owns a row: 16
// for rows of up to 128 features, a wavefront up to 1024, above that a workgroup.
// The gradient of the weight is a sum over all rows: each workgroup adds its own in
// registers, writes one row of sums, and a second kernel adds those in a fixed order.
//
// Everything is float32 until the one rounding to the output's type; an 8-bit value
// is the float32 output over its scale, rounded to nearest even.
//
// Measured, bf16 with the residual: 16384 rows of 768 features, 101 MB: forward
// 16 us (6.3 TB/s; a copy of as many bytes 15.7 us), gradient 20 + 4 us (4.1 TB/s);
// 4099 rows of 2048 to E4M3 by groups of 128, 59 MB: 14 us (4.2 TB/s).
#include "lbi_block.hpp"

namespace lbi {
namespace {

enum : int { kPlain = 0, kE4M3 = 1, kInt8 = 2 };

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
template <int LANES> __device__ __forceinline__ uint32_t row_max(uint32_t v, float *red, int parity)
{
    v = lanes_max<(LANES < 64 ? LANES : 64)>(v);
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64;
        uint32_t *r = (uint32_t *)red + parity * W;
        if ((threadIdx.x & 63) == 0)
            r[threadIdx.x >> 6] = v;
        __syncthreads();
        v = r[0];
#pragma unroll
        for (int w = 1; w < W; ++w)
            v = umax(v, r[w]);
    }
    return v;
}

template <int FMT> __device__ __forceinline__ uint32_t quantize4(const float *v, float scale)
{
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        constexpr float top = FMT == kE4M3 ? 448.f : 127.f;
        x[i] = v[i] / scale;
        // the quotient may round past the largest value; NaN passes through
        x[i] = x[i] > top ? top : (x[i] < -top ? -top : x[i]);
    }
    if constexpr (FMT == kE4M3) {
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], r, true);
    } else {
        uint32_t r = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r |= ((uint32_t)(int)rintf(x[i]) & 0xFFu) << (8 * i);
        return r;
    }
}

// The scale of a group from the bits of its largest |out|, and what its values are
// divided by.  Unsigned comparison of the bits ranks infinity and NaN above every
// number.
template <int FMT> __device__ __forceinline__ float scale_of(uint32_t top, float *by)
{
    const float scale = bitsf(top) * (FMT == kE4M3 ? 1.f / 448.f : 1.f / 127.f);
    if (top >= 0x7F800000u) {
        *by = bitsf(0x7FC00000u);
        return *by;
    }
    if (scale < 1.17549435e-38f) {
        *by = INFINITY;  // every value becomes 0
        return 1.f;
    }
    *by = scale;
    return scale;
}

template <typename X, typename R, int LANES, int NV, int FMT>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rms_kernel(const NormArgs a)
{
    constexpr int ROWS = LANES < 256 ? 256 / LANES : 1;
    __shared__ float red[LANES > 64 ? 2 * LANES / 64 : 1];
    __shared__ float red_max[LANES > 64 ? 2 * LANES / 64 : 1];
    const int lane = threadIdx.x % LANES;
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    const float over_D = 1.f / (float)a.D;
    int col[NV], left[NV];
    float w[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        col[j] = (j * LANES + lane) * 8;
        left[j] = a.D - col[j];
        load_some<8>(a.weight + col[j], left[j], w[j]);
    }
    int parity = 0;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; row < a.T; row += stride) {
        float s[NV][8];
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
        float sum[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                sum[0] += s[j][i] * s[j][i];
        row_sum<LANES>(sum, red, parity);
        const float r = rsqrtf(sum[0] * over_D + a.eps);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s[j][i] = s[j][i] * r * w[j][i];
        if constexpr (FMT == kPlain) {
            X *o = (X *)a.out + row * a.ld_out;
#pragma unroll
            for (int j = 0; j < NV; ++j)
                store_some<8>(o + col[j], left[j], s[j]);
        } else {
            uint32_t top[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                top[j] = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    top[j] = umax(top[j], fbits(s[j][i]) & 0x7FFFFFFFu);
            }
            float by[NV];
            float *scales = a.scales + row * a.ngroups;
            if (a.group == 0) {
                uint32_t m = top[0];
#pragma unroll
                for (int j = 1; j < NV; ++j)
                    m = umax(m, top[j]);
                m = row_max<LANES>(m, red_max, parity);
                const float scale = scale_of<FMT>(m, &by[0]);
#pragma unroll
                for (int j = 1; j < NV; ++j)
                    by[j] = by[0];
                if (lane == 0)
                    scales[0] = scale;
            } else {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    uint32_t m = lanes_max<4>(top[j]);
                    if (a.group >= 64)
                        m = umax(m, fbits(xchg<7>(bitsf(m))));
                    if (a.group >= 128)
                        m = umax(m, fbits(xchg<8>(bitsf(m))));
                    const float scale = scale_of<FMT>(m, &by[j]);
                    if (left[j] > 0 && (col[j] & (a.group - 1)) == 0)
                        scales[col[j] / a.group] = scale;
                }
            }
            uint8_t *o = (uint8_t *)a.out + row * a.ld_out;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const uint32_t q0 = quantize4<FMT>(s[j], by[j]);
                const uint32_t q1 = quantize4<FMT>(s[j] + 4, by[j]);
                if (left[j] >= 8) {
                    typedef u2 u2_byte __attribute__((aligned(1)));
                    *(u2_byte *)(o + col[j]) = u2{q0, q1};
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < left[j])
                            o[col[j] + i] = (uint8_t)((i < 4 ? q0 : q1) >> (8 * (i & 3)));
                }
            }
        }
        parity ^= 1;
    }
}

template <typename X, typename R, int LANES, int NV>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rms_backward_kernel(const NormArgs a)
{
    constexpr int ROWS = LANES < 256 ? 256 / LANES : 1;
    __shared__ float red[LANES > 64 ? 4 * LANES / 64 : 1];
    const int lane = threadIdx.x % LANES;
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    const float over_D = 1.f / (float)a.D;
    int col[NV], left[NV];
    float w[NV][8], dw[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        col[j] = (j * LANES + lane) * 8;
        left[j] = a.D - col[j];
        load_some<8>(a.weight + col[j], left[j], w[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            dw[j][i] = 0.f;
    }
    int parity = 0;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; row < a.T; row += stride) {
        float s[NV][8], g[NV][8], d[NV][8];
        const R *sp = (const R *)a.s + row * a.ld_s;
        const X *gp = (const X *)a.x + row * a.ld_x;
        const R *dp = a.residual ? (const R *)a.residual + row * a.ld_residual : nullptr;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            load_some<8>(sp + col[j], left[j], s[j]);
            load_some<8>(gp + col[j], left[j], g[j]);
            load_some<8>(dp ? dp + col[j] : dp, dp ? left[j] : 0, d[j]);
        }
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum[0] += s[j][i] * s[j][i];
                sum[1] += s[j][i] * (g[j][i] * w[j][i]);
            }
        row_sum<LANES>(sum, red, parity);
        const float r = rsqrtf(sum[0] * over_D + a.eps);
        const float m = sum[1] * r * over_D;  // mean(g n)
        R *o = (R *)a.out + row * a.ld_out;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float n = s[j][i] * r;
                dw[j][i] += g[j][i] * n;
                d[j][i] += r * (g[j][i] * w[j][i] - n * m);
            }
            store_some<8>(o + col[j], left[j], d[j]);
        }
        parity ^= 1;
    }
    if (!a.partial)
        return;
    float *part = a.partial + (int64_t)blockIdx.x * a.D;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            store_some<8>(part + col[j], left[j], dw[j]);
    } else {
        __shared__ float sums[ROWS][NV * LANES * 8];
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                sums[threadIdx.x / LANES][col[j] + i] = dw[j][i];
        __syncthreads();
        for (int c = threadIdx.x; c < a.D; c += 256) {
            float v = sums[0][c];
#pragma unroll
            for (int r = 1; r < ROWS; ++r)
                v += sums[r][c];
            part[c] = v;
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
// and up to 61 in the gradient, and a wavefront instead costs rows of 2048 up to 24 forward.
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

template <typename X, typename R, int FMT>
hipError_t forward(const NormArgs &a, hipStream_t stream)
{
    const Shape s = shape_of(a.D);
    const dim3 grid((unsigned)block_count(a.T, s.rows, kBlocks)), block(s.lanes < 256 ? 256 : s.lanes);
    return by_shape(s, [&](auto lanes, auto nv) {
        rms_kernel<X, R, decltype(lanes)::value, decltype(nv)::value, FMT>
            <<<grid, block, 0, stream>>>(a);
        return hipGetLastError();
    });
}
template <int FMT>
hipError_t forward_types(const NormArgs &a, bool bf16, bool residual_bf16, hipStream_t stream)
{
    if (bf16)
        return residual_bf16 ? forward<bf16_bits, bf16_bits, FMT>(a, stream)
                             : forward<bf16_bits, float, FMT>(a, stream);
    return residual_bf16 ? forward<float, bf16_bits, FMT>(a, stream)
                         : forward<float, float, FMT>(a, stream);
}
template <typename X, typename R> hipError_t backward(const NormArgs &a, hipStream_t stream)
{
    const Shape s = shape_of(a.D);
    const dim3 grid((unsigned)norm_partial_rows(a.T, a.D)), block(s.lanes < 256 ? 256 : s.lanes);
    return by_shape(s, [&](auto lanes, auto nv) {
        rms_backward_kernel<X, R, decltype(lanes)::value, decltype(nv)::value>
            <<<grid, block, 0, stream>>>(a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs &a, bool bf16, bool residual_bf16, hipStream_t stream)
{
    return forward_types<kPlain>(a, bf16, residual_bf16, stream);
}

hipError_t launch_rms_norm_q8(const NormArgs &a, bool int8, bool bf16, bool residual_bf16,
                              hipStream_t stream)
{
    return int8 ? forward_types<kInt8>(a, bf16, residual_bf16, stream)
                : forward_types<kE4M3>(a, bf16, residual_bf16, stream);
}

int64_t norm_partial_rows(int64_t T, int32_t D)
{
    const int rows = shape_of(D).rows;
    const int64_t n = block_count(T, rows, kBackwardBlocks);
    // four rows a workgroup at least where that leaves one a CU: each writes a row of sums
    const int64_t most = (T + 3) / 4 > 256 ? (T + 3) / 4 : 256;
    return n < most ? n : most;
}

hipError_t launch_rms_norm_backward(const NormArgs &a, float *dweight, bool bf16,
                                    bool residual_bf16, hipStream_t stream)
{
    if (a.T > 0) {
        const hipError_t e =
            bf16 ? (residual_bf16 ? backward<bf16_bits, bf16_bits>(a, stream)
                                  : backward<bf16_bits, float>(a, stream))
                 : (residual_bf16 ? backward<float, bf16_bits>(a, stream)
                                  : backward<float, float>(a, stream));
        if (e != hipSuccess)
            return e;
    }
    if (!dweight)
        return hipSuccess;
    return sum_rows(a.partial, a.T > 0 ? norm_partial_rows(a.T, a.D) : 0, a.D, a.D,
                    ToVector{dweight}, stream);
}

}  // namespace lbi
