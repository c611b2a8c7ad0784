// Device code shared by the forward and gradient kernels of linear attention: tiles of tokens in
// LDS, matrix operands from them in both orientations, a head's state in registers.
//
// One layout serves float32 and bf16.  An operand covers 32 values k of the summed index; lane
// (row c = lane & 15, group g = lane >> 4) holds k = 16 u + 4 g + r for u = 0, 1 and r = 0 .. 3.
// The sum over k does not mind the order, both operands have the same, and this one is that of
// two stacked 16 x 16 results: column c, rows 4 g + r.  So a state that is accumulated in
// registers is an operand as it stands, without a trip through LDS.
#ifndef LBI_ATTENTION_HPP
#define LBI_ATTENTION_HPP

#include "lbi_block.hpp"
#include "lbi_linear_internal.h"

namespace lbi {
namespace {

typedef short s4 __attribute__((ext_vector_type(4)));

// ---- matrix operands

// Tiles of bf16 in LDS have the two halves of every 16 values exchanged in rows 8 .. 15 of 16, at
// a stride of 32 bytes more than their values: 32 lanes that read 8 bytes each, of rows or of columns,
// then name all 64 banks once.  Stores of rows and reads of columns have no conflicts (ends_kernel has
// nothing else, and the counter is 0 there); the walks, which also read rows and store p and e, have
// them in 40 per cent of their LDS cycles (64 and 64).  Float32 tiles lie as they are.
template <typename T> __device__ __forceinline__ int swapped(int row)
{
    return sizeof(T) == 2 ? row & 8 : 0;
}
template <typename T> constexpr int tile_stride(int values) { return values + (sizeof(T) == 2 ? 16 : 4); }
// Where this lane's four values 4 g .. of 16 lie in row c of 16.
template <typename T> __device__ __forceinline__ int lane_quad()
{
    return 4 * (threadIdx.x >> 4 & 3) ^ swapped<T>(threadIdx.x & 15);
}

template <typename T> struct Frag;
template <> struct Frag<bf16_bits> {
    u4 w;  // pairs: k = 4 g + (0, 1), (2, 3), 16 + 4 g + (0, 1), (2, 3)

    // Of a tile [row][k]: lane c takes row `row0` + c.
    __device__ __forceinline__ void rows(const bf16_bits *m, int stride, int row0, int k0)
    {
        const int c = threadIdx.x & 15;
        const bf16_bits *p = m + (row0 + c) * stride + k0 + lane_quad<bf16_bits>();
        const u2 a = *(const u2 *)p, b = *(const u2 *)(p + 16);
        w = u4{a.x, a.y, b.x, b.y};
    }
    // Of a tile [k][col]: lane c takes column `col0` + c.  The hardware's transposing read: sixteen
    // lanes give the addresses of 4 rows of 16 values, four lanes a row, and get a column of 4 each.
    __device__ __forceinline__ void cols(const bf16_bits *m, int stride, int k0, int col0)
    {
        const int c = threadIdx.x & 15, g = threadIdx.x >> 4 & 3;
        const bf16_bits *p = m + (k0 + 4 * g + (c >> 2)) * stride + col0 + (4 * (c & 3) ^ (4 * g & 8));
        typedef __attribute__((address_space(3))) s4 lds_s4;
        const u2 a = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)p));
        const u2 b = __builtin_bit_cast(
            u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(p + 16 * stride)));
        w = u4{a.x, a.y, b.x, b.y};
    }
    __device__ __forceinline__ void unpack(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bitsf(w[i] << 16);
            x[2 * i + 1] = bitsf(w[i] & kHighHalf);
        }
    }
    __device__ __forceinline__ void pack(const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = narrow_pair(x[2 * i], x[2 * i + 1]);
    }
};
template <> struct Frag<float> {
    float v[8];

    __device__ __forceinline__ void rows(const float *m, int stride, int row0, int k0)
    {
        const int lane = threadIdx.x & 63;
        const float *p = m + (row0 + (lane & 15)) * stride + k0 + 4 * (lane >> 4);
        const f4 a = *(const f4 *)p, b = *(const f4 *)(p + 16);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            v[r] = a[r];
            v[4 + r] = b[r];
        }
    }
    __device__ __forceinline__ void cols(const float *m, int stride, int k0, int col0)
    {
        const int lane = threadIdx.x & 63;
        const float *p = m + (k0 + 4 * (lane >> 4)) * stride + col0 + (lane & 15);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            v[r] = p[r * stride];
            v[4 + r] = p[(16 + r) * stride];
        }
    }
    __device__ __forceinline__ void unpack(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = v[i];
    }
    __device__ __forceinline__ void pack(const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = x[i];
    }
};

// acc[row of A][row of B] += sum over k; lane: column c = row of B, rows 4 g + r of A.
__device__ __forceinline__ void mma(f4 &acc, const Frag<bf16_bits> &a, const Frag<bf16_bits> &b)
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.w),
                                                  __builtin_bit_cast(bf16x8, b.w), acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(f4 &acc, const Frag<float> &a, const Frag<float> &b)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], acc, 0, 0, 0);
}

// A float32 operand.  For the bf16 matrix cores it is a sum of bf16 values, for one product each:
// three are the value itself (what two round to nearest leave has at most 8 significant bits) and
// go into states, which are results in float32; two leave at most 2^-16 of it, a random rounding,
// and take a state into the outputs' and the values' gradients' products with tokens.
template <typename T, int PARTS> struct Wide;
template <int PARTS> struct Wide<bf16_bits, PARTS> {
    Frag<bf16_bits> part[PARTS];
    __device__ __forceinline__ void pack(const float (&x)[8])
    {
        float rest[8], h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            rest[i] = x[i];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            part[p].pack(rest);
            if (p + 1 < PARTS) {
                part[p].unpack(h);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    rest[i] -= h[i];
            }
        }
    }
};
template <int PARTS> struct Wide<float, PARTS> {
    Frag<float> part[1];
    __device__ __forceinline__ void pack(const float (&x)[8]) { part[0].pack(x); }
};
template <typename T, int PARTS>
__device__ __forceinline__ void mma(f4 &acc, const Wide<T, PARTS> &a, const Frag<T> &b)
{
#pragma unroll
    for (int p = (sizeof(T) == 2 ? PARTS : 1) - 1; p >= 0; --p)
        mma(acc, a.part[p], b);
}
template <typename T, int PARTS>
__device__ __forceinline__ void mma(f4 &acc, const Frag<T> &a, const Wide<T, PARTS> &b)
{
#pragma unroll
    for (int p = (sizeof(T) == 2 ? PARTS : 1) - 1; p >= 0; --p)
        mma(acc, a, b.part[p]);
}
template <typename T, int PARTS>
__device__ __forceinline__ void pack_tiles(Wide<T, PARTS> &w, const f4 &a, const f4 &b)
{
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    w.pack(x);
}

// ---- decays

// log2 of a head's factor: NaN where there is none (above 0), and a number that makes every power
// but the 0th vanish for -infinity.
__device__ __forceinline__ float log2_decay(const float *log_decay, int h)
{
    const float x = log_decay[h];
    return x <= 0.f ? fmaxf(x * kLog2e, -16384.f) : bitsf(0x7FC00000u);
}
// a^n
__device__ __forceinline__ float power(float l2, float n) { return __builtin_amdgcn_exp2f(n * l2); }

// ---- tiles of tokens in LDS

// Kernels come in two forms.  FULL: a head's keys and values fill the tiles' widths, so whole vectors
// are loaded and stored; otherwise every vector may end early, and the code for that is several times
// as long as the rest.

// Rows of a token tensor on their way into a tile [C][tile_stride(W)]: `values` of a head of each
// of n <= C tokens, zeros behind them.  Loads stay in flight until put().
template <typename T, int C, int W, bool FULL> struct TileLoad {
    static constexpr int COUNT = C * W / 2048, STEP = 2048 / W;  // rows between a thread's pieces
    Raw<T, 8> r[COUNT];

    __device__ __forceinline__ static int row() { return threadIdx.x / (W / 8); }
    __device__ __forceinline__ static int col() { return threadIdx.x % (W / 8) * 8; }
    // p, ld and n are the same in all threads; n > 0
    __device__ __forceinline__ void load(const T *p, int64_t ld, int n, int values)
    {
        p = uniform_pointer(p);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int at = row() + i * STEP;
            const uint32_t bytes = (uint32_t)((at < n ? at : 0) * (int)ld + col()) * (uint32_t)sizeof(T);
            if constexpr (FULL) {
                r[i].load(lane_address(p, bytes), 8);
                r[i].keep(at < n);
            } else {
                r[i].load(lane_address(p, bytes), at < n ? values - col() : 0);
            }
        }
    }
    // True where a value is infinite or NaN.
    __device__ __forceinline__ bool put(T *m) const
    {
        if constexpr (sizeof(T) == 2) {
            typedef unsigned short h2 __attribute__((ext_vector_type(2)));
            typedef short i2 __attribute__((ext_vector_type(2)));
            h2 high = {0, 0};  // largest bits of negative values
            i2 low = {0, 0};   // and of positive ones
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int at = row() + i * STEP;
                *(u4 *)(m + at * tile_stride<T>(W) + (col() ^ swapped<T>(at))) =
                    u4{r[i].w[0], r[i].w[1], r[i].w[2], r[i].w[3]};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    high = __builtin_elementwise_max(high, __builtin_bit_cast(h2, r[i].w[k]));
                    low = __builtin_elementwise_max(low, __builtin_bit_cast(i2, r[i].w[k]));
                }
            }
            return high.x >= 0xFF80 || high.y >= 0xFF80 || low.x >= 0x7F80 || low.y >= 0x7F80;
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                T *to = m + (row() + i * STEP) * tile_stride<T>(W) + col();
                *(f4 *)to = f4{r[i].v[0], r[i].v[1], r[i].v[2], r[i].v[3]};
                *(f4 *)(to + 4) = f4{r[i].v[4], r[i].v[5], r[i].v[6], r[i].v[7]};
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    top = umax(top, fbits(r[i].v[k]) & 0x7FFFFFFFu);
            }
            return top >= 0x7F800000u;
        }
    }
};
// A barrier, and whether any thread of the workgroup said `bad`.
__device__ __forceinline__ bool any_bad(bool bad, int *flags)
{
    const bool wave = __ballot(bad) != 0;
    if ((threadIdx.x & 63) == 0)
        flags[threadIdx.x >> 6] = wave;
    __syncthreads();
    return (flags[0] | flags[1] | flags[2] | flags[3]) != 0;
}

// ---- a head's state

// The state [DK][DV] of a head in registers: wavefront w has columns w DV / 4 .. of it, in 16 x 16
// results.  (With DK and DV exchanged: its transpose.)
template <typename T, int DK, int DV, bool FULL> struct State {
    static constexpr int KT = DK / 16, VT = DV / 64;
    f4 s[KT][VT];

    __device__ __forceinline__ static int column(int c)
    {
        return (threadIdx.x >> 6) * (DV / 4) + c * 16;
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int c = 0; c < VT; ++c)
                s[k][c] = f4{0.f, 0.f, 0.f, 0.f};
    }
    // f(value, its address) for the values that the head has; p: [dk][dv], row and col the distances
    // of neighbours.
    template <typename P, typename F>
    __device__ __forceinline__ void each(P *p, int dk, int dv, int row, int col, F &&f)
    {
        const int lane = threadIdx.x & 63, i0 = 4 * (lane >> 4), j0 = column(0) + (lane & 15);
        p = uniform_pointer(p);
        const uint32_t base = (uint32_t)(i0 * row + j0 * col) * 4;
        const bool whole = FULL || (dk == DK && dv == DV);
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int c = 0; c < VT; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (whole || (i0 < dk - 16 * k - r && j0 < dv - 16 * c)) {
                        float x = s[k][c][r];
                        f(x, lane_address(p + ((16 * k + r) * row + 16 * c * col), base));
                        s[k][c][r] = x;
                    }
    }
    // From memory; NULL: zeros.
    __device__ __forceinline__ void load(const float *p, int dk, int dv, int row, int col)
    {
        zero();
        if (p)
            each(p, dk, dv, row, col, [](float &x, const float *q) { x = *q; });
    }
    __device__ __forceinline__ void store(float *p, int dk, int dv)
    {
        each(p, dk, dv, dv, 1, [](float &x, float *q) { *q = x; });
    }
    // s = fade s + sum over the tile's tokens of a_t (w_t b_t)^T, a [C][DK], b [C][DV];
    // w[8 kb + 4 u + r]: the weight of token 32 kb + 16 u + 4 g + r.
    template <int C>
    __device__ __forceinline__ void update(const T *a, const T *b, const float (&w)[C / 4],
                                           float fade)
    {
#pragma unroll
        for (int c = 0; c < VT; ++c) {
            Wide<T, 3> wb[C / 32];
#pragma unroll
            for (int kb = 0; kb < C / 32; ++kb) {
                Frag<T> f;
                f.cols(b, tile_stride<T>(DV), 32 * kb, column(c));
                float x[8];
                f.unpack(x);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    x[i] *= w[8 * kb + i];
                wb[kb].pack(x);
            }
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                f4 acc = s[k][c] * fade;
#pragma unroll
                for (int kb = 0; kb < C / 32; ++kb) {
                    Frag<T> f;
                    f.cols(a, tile_stride<T>(DK), 32 * kb, 16 * k);
                    mma(acc, f, wb[kb]);
                }
                s[k][c] = acc;
            }
        }
    }
};

// Weights of a tile's tokens 0 .. n - 1: what is left of token t at the tile's end, a^(n-1-t), or
// what of the state before it reaches it, scale a^(t+1).
template <int C> __device__ __forceinline__ void to_end(float (&w)[C / 4], float l2, int n)
{
    const int g = (threadIdx.x >> 4) & 3;
#pragma unroll
    for (int i = 0; i < C / 4; ++i) {
        const int t = 16 * (i / 4) + 4 * g + i % 4;
        w[i] = t < n ? power(l2, (float)(n - 1 - t)) : 0.f;
    }
}
template <int C>
__device__ __forceinline__ void from_start(float (&w)[C / 4], float l2, int n, float scale)
{
    const int g = (threadIdx.x >> 4) & 3;
#pragma unroll
    for (int i = 0; i < C / 4; ++i) {
        const int t = 16 * (i / 4) + 4 * g + i % 4;
        w[i] = t < n ? power(l2, (float)(t + 1)) * scale : 0.f;
    }
}

// ---- ranges of tokens

__device__ __forceinline__ Sequences sequences_of(const lbi_attention_inputs &in)
{
    return {in.offsets, in.T, in.sequences, in.sequences > 0 ? in.T / in.sequences : 0};
}
// The rows first .. end - 1 of a range.
struct Rows {
    int64_t first, end;
    __device__ __forceinline__ Rows(const AttentionArgs &a, int64_t range)
    {
        if (a.cut.per_sequence > 0) {
            const int64_t len = a.in.T / a.in.sequences, seq = range / a.cut.per_sequence;
            first = seq * len + range % a.cut.per_sequence * a.cut.tokens;
            end = first + a.cut.tokens;
            if (end > (seq + 1) * len) end = (seq + 1) * len;
        } else {
            first = range * a.cut.tokens;
            end = first + a.cut.tokens;
            if (end > a.in.T) end = a.in.T;
        }
    }
};

// 4 consecutive values of a token's row
template <typename T, bool FULL = false>
__device__ __forceinline__ void store4(T *p, int left, const f4 &v)
{
    const float x[4] = {v.x, v.y, v.z, v.w};
    store_some<4>(p, FULL ? 4 : left, x);
}
// ... into a tile
__device__ __forceinline__ void put4(bf16_bits *p, const f4 &v)
{
    *(u2 *)p = u2{narrow_pair(v.x, v.y), narrow_pair(v.z, v.w)};
}
__device__ __forceinline__ void put4(float *p, const f4 &v) { *(f4 *)p = v; }
// ... out of a tile
__device__ __forceinline__ f4 get4(const bf16_bits *p)
{
    const u2 a = *(const u2 *)p;
    return f4{bitsf(a.x << 16), bitsf(a.x & kHighHalf), bitsf(a.y << 16), bitsf(a.y & kHighHalf)};
}
__device__ __forceinline__ f4 get4(const float *p) { return *(const f4 *)p; }

// The 16 x 16 tiles (row, column) of a tile's C x C products of queries and keys that are needed,
// dealt to the wavefronts: f(which, row, column) for column <= row, and for those beside the
// diagonal that operands of 32 read as zeros (column = row + 1, row even).
template <int C> constexpr int kCausalTiles = C == 64 ? 3 : 1;  // of a wavefront
template <int C, typename F> __device__ __forceinline__ void causal_tiles(F &&f)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int at = 0; at < kCausalTiles<C>; ++at)
        f(at, at == 0 ? wave >> 1 : at + 1, at == 0 ? wave & 1 : wave);
}
// scale a^(i-j) at this lane's places of those tiles, 0 for j > i.
template <int C>
__device__ __forceinline__ void causal_fade(f4 (&fade)[kCausalTiles<C>], float l2, float scale)
{
    causal_tiles<C>([&](int at, int it, int jt) {
        const int lag = 16 * (it - jt) + (threadIdx.x & 15) - 4 * (threadIdx.x >> 4 & 3);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            fade[at][r] = lag >= r ? power(l2, (float)(lag - r)) * scale : 0.f;
    });
}

// Between phases that take the same operands from LDS: they are loaded again rather than kept.
__device__ __forceinline__ void phase()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Calls f(type, DK, DV, FULL) with the storage type and the tiles' widths for the head's.
template <typename F> hipError_t by_head(const lbi_attention_inputs &in, F &&f)
{
    using W64 = std::integral_constant<int, 64>;
    using W128 = std::integral_constant<int, 128>;
    auto full = [&](auto type, auto dk, auto dv) {
        if (in.DK == decltype(dk)::value && in.DV == decltype(dv)::value)
            return f(type, dk, dv, std::true_type{});
        return f(type, dk, dv, std::false_type{});
    };
    auto widths = [&](auto type) {
        if (in.DK <= 64)
            return in.DV <= 64 ? full(type, W64{}, W64{}) : full(type, W64{}, W128{});
        return in.DV <= 64 ? full(type, W128{}, W64{}) : full(type, W128{}, W128{});
    };
    return in.dt == LBI_BF16 ? widths(bf16_bits{}) : widths(float{});
}

}  // namespace
}  // namespace lbi

#endif  // LBI_ATTENTION_HPP
