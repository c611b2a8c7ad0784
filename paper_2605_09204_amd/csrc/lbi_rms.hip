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
// is the float32 output over its scale, rounded to nearest even, from a sum in a stated
// order (sum_in_order).
//
// Measured, bf16 with the residual: 16384 rows of 768 features, 101 MB: forward
// 16 us (6.3 TB/s; a copy of as many bytes 15.7 us), gradient 20 + 4 us (4.1 TB/s);
// 4099 rows of 2048 to E4M3 by groups of 128, 59 MB: 14.5 us (4.1 TB/s; one less with the squares
// added in registers, in no stated order).
#include "lbi_norm_rows.hpp"

namespace lbi {
namespace {

enum : int { kE4M3, kInt8 };

template <int LANES> __device__ __forceinline__ uint32_t row_max(uint32_t v, float *red)
{
    v = lanes_max<(LANES < 64 ? LANES : 64)>(v);
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64;
        uint32_t *r = (uint32_t *)red;
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

template <typename X, typename R, int LANES, int NV>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rms_kernel(const NormArgs a)
{
    constexpr int ROWS = LANES < 256 ? 256 / LANES : 1;
    __shared__ float red[LANES > 64 ? 2 * LANES / 64 : 1];
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
        load_sum<X, R, NV>(a, row, col, left, s);
        float sum[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                sum[0] += s[j][i] * s[j][i];
        row_sum<LANES>(sum, red, parity);
        const float r = rsqrtf(sum[0] * over_D + a.eps);
        X *o = (X *)a.out + row * a.ld_out;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s[j][i] = s[j][i] * r * w[j][i];
            store_some<8>(o + col[j], left[j], s[j]);
        }
        parity ^= 1;
    }
}

// The 8-bit form's sum of squares.  A quotient in the middle between two 8-bit values goes
// by the last bit of this sum, so its order is part of the interface: the one in which the
// usual tensor operations add a dense float32 row, whose bytes these then are.
//
// Rows below 128 features: sum l of L = min(64, the largest power of two up to D) is
// x_l + x_{l+L}.  Wider ones: the row's vectors of four, which begin where t D + d is a
// multiple of four; 64 lanes (32 below 256 features, 512 above 8128) take one each in turn, a
// lane's four sums grow along the row and are then added in order.  What lies ahead of the
// first vector or after the last joins the first sum of lanes (t D mod 4) .. 3 and 0 .. 2.  The
// lanes' sums are added pairwise, neighbours first, up to 64 of them; what that leaves of 512
// by halves, the first with the fifth.
//
// The squares are exchanged in LDS: element d lies at d + shift, shift = t D mod 4, which
// puts the vectors at multiples of four.
struct RowOrder {
    int shift, first, vectors, tail;  // first: where the vectors begin in LDS
    __device__ __forceinline__ RowOrder(int64_t row, int D)
    {
        shift = D < 128 ? 0 : (int)((row * D) & 3);
        const int head = shift ? 4 - shift : 0;
        first = shift ? 4 : 0;
        vectors = (D - head) >> 2;
        tail = (D - head) & 3;
    }
};
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// By a wavefront; WIDTH: most features.
template <int WIDTH>
__device__ __forceinline__ float sum_in_order(const float *sq, int D, int64_t row)
{
    const int lane = threadIdx.x & 63;
    if (D < 128) {
        const int L = D >= 64 ? 64 : 1 << (31 - __clz(D));
        const float more = lane + L < D ? sq[lane + L] : 0.f;
        return lanes_sum<64>(lane < L ? sq[lane] + more : 0.f);
    }
    const RowOrder o(row, D);
    const int L = D < 256 ? 32 : 64;
    f4 a = {0.f, 0.f, 0.f, 0.f};
    if (lane >= o.shift && lane < o.first)
        a.x = sq[lane];
#pragma unroll
    for (int v = lane, k = 0; k < (WIDTH + 255) / 256; v += L, ++k) {
        const bool there = lane < L && v < o.vectors;
        const f4 q = *(const f4 *)(sq + (there ? o.first + 4 * v : 0));
        if (there)
            a += q;
    }
    if (lane < o.tail)
        a.x += sq[o.first + 4 * o.vectors + lane];
    return lanes_sum<64>(((a.x + a.y) + a.z) + a.w);
}
// By a workgroup, the four sums of a lane in four threads side by side; MANY: 512 lanes, eight
// a thread (registers for them cost narrower rows a third of their speed).
template <int WIDTH, bool MANY>
__device__ __forceinline__ float sum_in_order_together(const float *sq, int D, int64_t row,
                                                       float (*red)[8])
{
    const int t = threadIdx.x;
    if (t < 256) {
        const RowOrder o(row, D);
        const bool head = (t & 3) == 0 && t >> 2 >= o.shift && t >> 2 < o.first;
        const bool tail = (t & 3) == 0 && t >> 2 < o.tail;
        const float before = head ? sq[t >> 2] : 0.f;
        const float after = tail ? sq[o.first + 4 * o.vectors + (t >> 2)] : 0.f;
        auto value = [&](int k) {
            const int i = t + 256 * k;
            const float q = sq[o.first + i];
            return i < 4 * o.vectors ? q : 0.f;
        };
        // over the quad in order (quad_perm broadcasts), then over the wavefront's 16 lanes
        auto wave = [&](float a, int m) {
            float s = ((dpp<0x00>(a) + dpp<0x55>(a)) + dpp<0xAA>(a)) + dpp<0xFF>(a);
            s += xchg<7>(s);
            s += xchg<8>(s);
            s = add_rows<16>(s, s);
            s = add_rows<32>(s, s);
            if ((t & 63) == 0)
                red[t >> 6][m] = s;
        };
        if constexpr (MANY) {
            float a[8] = {before};
#pragma unroll
            for (int k = 0; k < WIDTH / 256; k += 8)
#pragma unroll
                for (int m = 0; m < 8; ++m)
                    a[m] += value(k + m);
            a[0] += after;
#pragma unroll
            for (int m = 0; m < 8; ++m)
                wave(a[m], m);
        } else {
            float a = before;
#pragma unroll 16
            for (int k = 0; k < WIDTH / 256; ++k)
                a += value(k);
            wave(a + after, 0);
        }
    }
    __syncthreads();
    auto sum = [&](int m) { return (red[0][m] + red[1][m]) + (red[2][m] + red[3][m]); };
    if constexpr (!MANY)
        return sum(0);
    else
        return ((sum(0) + sum(4)) + (sum(2) + sum(6))) + ((sum(1) + sum(5)) + (sum(3) + sum(7)));
}
// 1 / sqrt(sum / D + eps), rounded to nearest: product and sum each by itself, and the
// hardware's root (one unit of the last place) with a Newton step whose residual 1 - m r^2 is
// exact to second order.  (One root in some 10^7 lies so near the middle that it goes the other
// way.)
__device__ __forceinline__ float reciprocal_root(float sum, float over_D, float eps)
{
#pragma clang fp contract(off)
    const float mean = sum * over_D;
    const float m = mean + eps, r = rsqrtf(m);
    const float h = m * r, low = fmaf(m, r, -h);
    const float e = fmaf(-h, r, 1.f) - low * r;
    return r > 0.f && r < INFINITY ? fmaf(0.5f * r, e, r) : r;
}

template <typename X, typename R, int LANES, int NV, int FMT, bool MANY>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rms_q8_kernel(const NormArgs a)
{
    constexpr int ROWS = LANES < 256 ? 256 / LANES : 1, WIDTH = LANES * NV * 8, PITCH = WIDTH + 4;
    __shared__ __align__(16) float squares[ROWS * PITCH];
    __shared__ float red[4][8];
    __shared__ float red_max[LANES > 64 ? LANES / 64 : 1];
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
    float *mine = squares + threadIdx.x / LANES * PITCH;
    for (int64_t base = (int64_t)blockIdx.x * ROWS; base < a.T; base += stride) {
        const int64_t row = base + threadIdx.x / LANES;
        const bool live = row < a.T;
        int there[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j)
            there[j] = live ? left[j] : 0;
        float s[NV][8];
        load_sum<X, R, NV>(a, row, col, there, s);
        const int shift = RowOrder(row, a.D).shift;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = s[j][i] * s[j][i];
            float *p = mine + col[j] + shift;
            if (shift == 0 && there[j] >= 8) {
                *(f4 *)p = f4{v[0], v[1], v[2], v[3]};
                *(f4 *)(p + 4) = f4{v[4], v[5], v[6], v[7]};
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < there[j])
                        p[i] = v[i];
            }
        }
        float sum = 0.f;
        if constexpr (LANES > 64) {
            __syncthreads();
            sum = sum_in_order_together<WIDTH, MANY>(squares, a.D, row, red);
        } else {
            // the rows of a wavefront, one after the other
            wave_sync();
            constexpr int PER_WAVE = 64 / LANES;
            const int first = (threadIdx.x >> 6) * PER_WAVE;
#pragma unroll
            for (int k = 0; k < PER_WAVE; ++k) {
                const float v =
                    sum_in_order<WIDTH>(squares + (first + k) * PITCH, a.D, base + first + k);
                if (PER_WAVE == 1 || (int)(threadIdx.x & 63) / LANES == k)
                    sum = v;
            }
            wave_sync();
        }
        const float r = reciprocal_root(sum, over_D, a.eps);
        uint32_t top[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            top[j] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[j][i] = s[j][i] * r * w[j][i];
                top[j] = umax(top[j], fbits(s[j][i]) & 0x7FFFFFFFu);
            }
        }
        float by[NV];
        float *scales = a.scales + row * a.ngroups;
        if (a.group == 0) {
            uint32_t m = top[0];
#pragma unroll
            for (int j = 1; j < NV; ++j)
                m = umax(m, top[j]);
            m = row_max<LANES>(m, red_max);
            const float scale = scale_of<FMT>(m, &by[0]);
#pragma unroll
            for (int j = 1; j < NV; ++j)
                by[j] = by[0];
            if (lane == 0 && live)
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
                if (there[j] > 0 && (col[j] & (a.group - 1)) == 0)
                    scales[col[j] / a.group] = scale;
            }
        }
        uint8_t *o = (uint8_t *)a.out + row * a.ld_out;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t q0 = quantize4<FMT>(s[j], by[j]);
            const uint32_t q1 = quantize4<FMT>(s[j] + 4, by[j]);
            if (there[j] >= 8) {
                typedef u2 u2_byte __attribute__((aligned(1)));
                *(u2_byte *)(o + col[j]) = u2{q0, q1};
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < there[j])
                        o[col[j] + i] = (uint8_t)((i < 4 ? q0 : q1) >> (8 * (i & 3)));
            }
        }
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

template <typename X, typename R> hipError_t forward(const NormArgs &a, hipStream_t stream)
{
    const Shape s = shape_of(a.D);
    const dim3 grid((unsigned)block_count(a.T, s.rows, kBlocks)), block(s.lanes < 256 ? 256 : s.lanes);
    return by_shape(s, [&](auto lanes, auto nv) {
        rms_kernel<X, R, decltype(lanes)::value, decltype(nv)::value><<<grid, block, 0, stream>>>(a);
        return hipGetLastError();
    });
}
template <typename X, typename R, int FMT> hipError_t forward_q8(const NormArgs &a, hipStream_t stream)
{
    const Shape s = shape_of(a.D);
    const dim3 grid((unsigned)block_count(a.T, s.rows, kBlocks)), block(s.lanes < 256 ? 256 : s.lanes);
    return by_shape(s, [&](auto lanes, auto nv) {
        constexpr int LANES = decltype(lanes)::value, NV = decltype(nv)::value;
        if constexpr (LANES * NV * 8 >= 8192) {
            if (LANES == 1024 || a.D > 8128) {
                rms_q8_kernel<X, R, LANES, NV, FMT, true><<<grid, block, 0, stream>>>(a);
                return hipGetLastError();
            }
        }
        if constexpr (LANES < 1024)
            rms_q8_kernel<X, R, LANES, NV, FMT, false><<<grid, block, 0, stream>>>(a);
        return hipGetLastError();
    });
}
template <int FMT>
hipError_t q8_types(const NormArgs &a, bool bf16, bool residual_bf16, hipStream_t stream)
{
    if (bf16)
        return residual_bf16 ? forward_q8<bf16_bits, bf16_bits, FMT>(a, stream)
                             : forward_q8<bf16_bits, float, FMT>(a, stream);
    return residual_bf16 ? forward_q8<float, bf16_bits, FMT>(a, stream)
                         : forward_q8<float, float, FMT>(a, stream);
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
    if (bf16)
        return residual_bf16 ? forward<bf16_bits, bf16_bits>(a, stream)
                             : forward<bf16_bits, float>(a, stream);
    return residual_bf16 ? forward<float, bf16_bits>(a, stream) : forward<float, float>(a, stream);
}

hipError_t launch_rms_norm_q8(const NormArgs &a, bool int8, bool bf16, bool residual_bf16,
                              hipStream_t stream)
{
    return int8 ? q8_types<kInt8>(a, bf16, residual_bf16, stream)
                : q8_types<kE4M3>(a, bf16, residual_bf16, stream);
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
