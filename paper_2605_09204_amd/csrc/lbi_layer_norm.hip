// Layer norm with the residual's addition, and its gradient.
//
//   s = x + residual,  n = (s - mean(s)) r,  r = 1 / sqrt(mean((s - mean)^2) + eps),
//   out = n weight + bias
//   ds = r (g - mean(g) - n mean(g n)) + dresidual,  g = dout weight
//   dweight = sum over rows of dout n,  dbias = sum over rows of dout
//
// As in the root-mean-square norm, a row is read once and stays in registers, its sums are
// formed over its lanes, and HBM is the bound.  The mean comes first, then the squares of the
// differences from it, so nothing cancels where the mean is far from zero; the differences'
// own mean, what the first one's rounding left, is taken off in the same sums.
// The mean is the row's first value and the mean of the distances from it: equal values, whose
// variance would otherwise be what roundings leave, have differences of exactly zero.  Terms are
// divided by D before they are added, so no sum but that of the squares leaves float32's range;
// where that one does, 1 / sqrt is 0 and the row gives its bias.
// Everything is float32 until the one rounding to the output's type.
//
// 16384 x 768 bf16 with a residual: 18.5 us (101 MB, 5.4 TB/s: a copy's rate).  The gradient at
// 12289 x 768 bf16 on a float32 stream (132 MB): 26 us and 4 for the parameters' sums, one row after
// the other at three wavefronts a SIMD.
#include "lbi_linear_internal.h"
#include "lbi_norm_rows.hpp"

namespace lbi {
namespace {

// The value of the row's first lane.  slot: LDS that the row's sums do not use.
template <int LANES> __device__ __forceinline__ float of_first_lane(float x, float *slot)
{
    if constexpr (LANES == 64) {
        return bitsf(__builtin_amdgcn_readfirstlane(fbits(x)));
    } else if constexpr (LANES < 64) {
        return __shfl(x, 0, LANES);
    } else {
        if (threadIdx.x == 0)
            *slot = x;
        __syncthreads();  // two more until the next row writes it
        return bitsf(__builtin_amdgcn_readfirstlane(fbits(*slot)));
    }
}

// s -> s - mean for the row's features, 0 behind them.  Halves keep the distances in range.
template <int LANES, int NV>
__device__ __forceinline__ void centre(float (&s)[NV][8], const int (&left)[NV], float over_D,
                                       float *red)
{
    const float first = of_first_lane<LANES>(s[0][0], red + (LANES > 64 ? LANES / 64 : 0));
    const float half = 0.5f * first;
    float sum[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            sum[0] = fmaf(i < left[j] ? fmaf(0.5f, s[j][i], -half) : 0.f, over_D, sum[0]);
    row_sum<LANES>(sum, red, 0);
    const float mean = fmaf(2.f, sum[0], first);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s[j][i] = i < left[j] ? s[j][i] - mean : 0.f;
}

// 1 / sqrt(var + eps) from the squares' sum and the differences' mean: 0 for an infinite sum (the
// square of the rest alone might be infinite too), NaN for a NaN and an infinite difference.
__device__ __forceinline__ float reciprocal_root(float squares, float over_D, float rest, float eps)
{
    const float var = fmaf(-rest, rest, squares * over_D);
    return rsqrtf((var < 0.f ? 0.f : var) + eps);
}

template <int NV>
__device__ __forceinline__ void load_vector(const float *p, const int (&col)[NV],
                                            const int (&left)[NV], float otherwise,
                                            float (&v)[NV][8])
{
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (p) {
            load_some<8>(p + col[j], left[j], v[j]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[j][i] = otherwise;
        }
    }
}

template <typename X, typename R, int LANES, int NV>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void layer_norm_kernel(const NormArgs a)
{
    constexpr int ROWS = LANES < 256 ? 256 / LANES : 1, W = LANES > 64 ? LANES / 64 : 1;
    __shared__ float red[4 * W];
    const int lane = threadIdx.x % LANES;
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    const float over_D = 1.f / (float)a.D;
    int col[NV], left[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        col[j] = (j * LANES + lane) * 8;
        left[j] = a.D - col[j];
    }
    float w[NV][8], b[NV][8];
    load_vector<NV>(a.weight, col, left, 1.f, w);
    load_vector<NV>(a.bias, col, left, 0.f, b);
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; row < a.T; row += stride) {
        float s[NV][8];
        load_sum<X, R, NV>(a, row, col, left, s);
        centre<LANES, NV>(s, left, over_D, red);
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum[0] = fmaf(s[j][i], over_D, sum[0]);
                sum[1] += s[j][i] * s[j][i];
            }
        row_sum<LANES>(sum, red, 1);
        const float rest = sum[0], r = reciprocal_root(sum[1], over_D, rest, a.eps);
        X *o = (X *)a.out + row * a.ld_out;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s[j][i] = (s[j][i] - rest) * r * w[j][i] + b[j][i];
            store_some<8>(o + col[j], left[j], s[j]);
        }
    }
}

template <typename X, typename R, int LANES, int NV>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void layer_norm_backward_kernel(
    const NormArgs a)
{
    constexpr int ROWS = LANES < 256 ? 256 / LANES : 1, W = LANES > 64 ? LANES / 64 : 1;
    // rows above 8192 features: the registers do not hold the sums of the parameters' gradients
    // beside a row, so each thread keeps its own in LDS (behind the row's sums: addresses past 64 KB
    // would take a register each)
    constexpr bool KEEP = LANES * NV < 2048;
    constexpr int SUMS = KEEP ? 0 : NV * LANES * 8;
    __shared__ __align__(16) float red[8 * W + 2 * SUMS];
    float *const kept[2] = {red + 8 * W, red + 8 * W + SUMS};
    const int lane = threadIdx.x % LANES;
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    const float over_D = 1.f / (float)a.D;
    int col[NV], left[NV];
    float w[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        col[j] = (j * LANES + lane) * 8;
        left[j] = a.D - col[j];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            dw[j][i] = db[j][i] = 0.f;
    }
    if constexpr (NV == 1)
        load_vector<NV>(a.weight, col, left, 1.f, w);
    if constexpr (!KEEP)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            store_all<8>(kept[0] + col[j], dw[j]);
            store_all<8>(kept[1] + col[j], db[j]);
        }
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
        if constexpr (NV > 1)  // two sums a feature beside it would leave room for fewer wavefronts
            load_vector<NV>(a.weight, col, left, 1.f, w);
        centre<LANES, NV>(s, left, over_D, red);
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float gw = g[j][i] * w[j][i];
                sum[0] = fmaf(s[j][i], over_D, sum[0]);
                sum[1] += s[j][i] * s[j][i];
                sum[2] += gw;
                sum[3] += gw * s[j][i];
            }
        row_sum<LANES>(sum, red, 1);
        const float rest = sum[0], r = reciprocal_root(sum[1], over_D, rest, a.eps);
        const float mean_g = sum[2] * over_D;
        // 0 with an r of 0, where the last sum may have left the range
        const float mean_gn = r > 0.f ? (sum[3] - rest * sum[2]) * r * over_D : 0.f;
        R *o = (R *)a.out + row * a.ld_out;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if constexpr (!KEEP) {
                load_some<8>(kept[0] + col[j], 8, dw[j]);
                load_some<8>(kept[1] + col[j], 8, db[j]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float n = (s[j][i] - rest) * r;
                dw[j][i] += g[j][i] * n;
                db[j][i] += g[j][i];
                d[j][i] += r * (g[j][i] * w[j][i] - mean_g - n * mean_gn);
            }
            store_some<8>(o + col[j], left[j], d[j]);
            if constexpr (!KEEP) {
                store_all<8>(kept[0] + col[j], dw[j]);
                store_all<8>(kept[1] + col[j], db[j]);
            }
        }
    }
    if (!a.partial)
        return;
    // this workgroup's row of sums: dweight, then dbias
    float *part = a.partial + (int64_t)blockIdx.x * 2 * a.D;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if constexpr (!KEEP) {
                load_some<8>(kept[0] + col[j], 8, dw[j]);
                load_some<8>(kept[1] + col[j], 8, db[j]);
            }
            store_some<8>(part + col[j], left[j], dw[j]);
            store_some<8>(part + a.D + col[j], left[j], db[j]);
        }
    } else {
        __shared__ float sums[ROWS][NV * LANES * 8];
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    sums[threadIdx.x / LANES][col[j] + i] = which ? db[j][i] : dw[j][i];
            __syncthreads();
            for (int c = threadIdx.x; c < a.D; c += 256) {
                float v = sums[0][c];
#pragma unroll
                for (int r = 1; r < ROWS; ++r)
                    v += sums[r][c];
                part[which * a.D + c] = v;
            }
        }
    }
}

struct ToWeightAndBias {
    float *weight, *bias;  // either may be NULL
    int32_t D;
    __device__ __forceinline__ void operator()(int64_t c, float v) const
    {
        float *to = c < D ? weight : bias;
        if (to)
            to[c < D ? c : c - D] = v;
    }
};

template <typename X, typename R>
hipError_t forward(const NormArgs &a, hipStream_t stream)
{
    const Shape s = shape_of(a.D);
    const dim3 grid((unsigned)block_count(a.T, s.rows, kBlocks)), block(s.lanes < 256 ? 256 : s.lanes);
    return by_shape(s, [&](auto lanes, auto nv) {
        layer_norm_kernel<X, R, decltype(lanes)::value, decltype(nv)::value>
            <<<grid, block, 0, stream>>>(a);
        return hipGetLastError();
    });
}
// Two sums a feature stay in registers, so rows above 4096 features get 1024 lanes.
Shape backward_shape(int32_t D)
{
    return D > 4096 && D <= 8192 ? Shape{1024, 1, 1} : shape_of(D);
}
template <typename X, typename R> hipError_t backward(const NormArgs &a, hipStream_t stream)
{
    const Shape s = backward_shape(a.D);
    const dim3 grid((unsigned)layer_norm_partial_rows(a.T, a.D)), block(s.lanes < 256 ? 256 : s.lanes);
    if (s.lanes == 1024 && s.nv == 1) {
        layer_norm_backward_kernel<X, R, 1024, 1><<<grid, block, 0, stream>>>(a);
        return hipGetLastError();
    }
    return by_shape(s, [&](auto lanes, auto nv) {
        constexpr int LANES = decltype(lanes)::value, NV = decltype(nv)::value;
        if constexpr (LANES != 256 || NV != 4)
            layer_norm_backward_kernel<X, R, LANES, NV><<<grid, block, 0, stream>>>(a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_layer_norm(const NormArgs &a, bool bf16, bool residual_bf16, hipStream_t stream)
{
    if (bf16)
        return residual_bf16 ? forward<bf16_bits, bf16_bits>(a, stream)
                             : forward<bf16_bits, float>(a, stream);
    return residual_bf16 ? forward<float, bf16_bits>(a, stream) : forward<float, float>(a, stream);
}

// As for the root-mean-square norm, but three workgroups a CU for rows of 513 to 4096 features: what
// the GPU holds at once above 1024 (registers); up to there it would hold four.
int64_t layer_norm_partial_rows(int64_t T, int32_t D)
{
    const Shape s = backward_shape(D);
    const int64_t n = norm_partial_rows(T, D);
    return s.nv > 1 && s.lanes < 1024 && n > 768 ? 768 : n;
}

hipError_t launch_layer_norm_backward(const NormArgs &a, float *dweight, float *dbias, bool bf16,
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
    if (!dweight && !dbias)
        return hipSuccess;
    return sum_rows(a.partial, a.T > 0 ? layer_norm_partial_rows(a.T, a.D) : 0, 2 * (int64_t)a.D,
                    2 * (int64_t)a.D, ToWeightAndBias{dweight, dbias, a.D}, stream);
}

}  // namespace lbi
