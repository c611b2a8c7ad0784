// Matrix products with bias, activation and residual in their epilogue, and what the gradient of
// one needs beside two more products.
//
//   out = act(x W^T + bias) + residual;   dz = dout act'(z), dx = dz W, dW = dz^T x
//
// The three differ in how the operands lie: the index that is summed runs along the rows of both
// (forward), of one (dx) or of none (dW).  A workgroup takes a BM x BN tile of the result, the
// operands pass through LDS as they lie, and the matrix instructions' operands are read from there
// straight or through the transposing read.
//
// bf16, 16384 x 768 onto 1536 takes 49 us (790 TFLOP/s), 58 with SiLU and z written; 4096^3 124 us
// (1110).  Between the barriers of two stages the matrix cores wait for LDS; a tile of 128 x 128, whose
// two stages take 64 KB of it, leaves two workgroups a CU, which fill each other's waits (of the 256
// registers that each lane then has they take 130 to 152).  float32 4096^3: 730 us (188),
// bound by the vector ALUs that split the operands beside the matrix cores.
#include "lbi_attention.hpp"
#include "lbi_dma.hpp"

namespace lbi {
namespace {

// ---- activations

template <int ACT> __device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == LBI_ACT_SILU)
        return silu(z);
    else if constexpr (ACT == LBI_ACT_GELU)
        return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    else
        return z;
}
template <int ACT> __device__ __forceinline__ float slope(float z)
{
    if constexpr (ACT == LBI_ACT_SILU)
        return silu_slope(z, sigmoid(z));
    else if constexpr (ACT == LBI_ACT_GELU)  // z times the normal density vanishes at the ends
        return 0.5f * (1.f + erff(z * 0.70710678118654752f)) +
               z * __builtin_amdgcn_exp2f(fmaxf(-0.5f * kLog2e * z * z, -200.f)) * 0.39894228040143268f;
    else
        return 1.f;
}

// ---- the product

// Operand of 32 values k from a tile in LDS: bf16 in their order, 8 g .. 8 g + 7 in lane group g.
template <typename T, bool COLS>
__device__ __forceinline__ void operand(Frag<T> &f, const T *m, int stride, int row0, int k0)
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (COLS) f.cols(m, stride, k0, row0);
        else f.rows(m, stride, row0, k0);
    } else if constexpr (COLS) {
        const int lane = threadIdx.x & 63, c = lane & 15;
        const T *p = m + (k0 + 8 * (lane >> 4) + (c >> 2)) * stride + row0 + 4 * (c & 3);
        typedef __attribute__((address_space(3))) s4 lds_s4;
        const u2 a = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)p));
        const u2 b = __builtin_bit_cast(
            u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(p + 4 * stride)));
        f.w = u4{a.x, a.y, b.x, b.y};
    } else {
        const int lane = threadIdx.x & 63;
        f.w = *(const u4 *)(m + (row0 + (lane & 15)) * stride + k0 + 8 * (lane >> 4));
    }
}

// What the matrix cores are given of an operand.  Float32 values go in as three bf16 values that
// add up to them: of the nine products of two such sums the six down to 2^-16 of the first are
// taken, which leaves what float32 products round away (the library's default arithmetic for
// float32), at 6 / 16 of the float32 matrix cores' time.
template <typename T> struct Factor;
template <> struct Factor<bf16_bits> {
    Frag<bf16_bits> f;
    __device__ __forceinline__ void set(const Frag<bf16_bits> &x) { f = x; }
};
template <> struct Factor<float> {
    Frag<bf16_bits> h, m, l;
    __device__ __forceinline__ void set(const Frag<float> &x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Split2 s = split_pair(x.v[2 * i], x.v[2 * i + 1]);
            h.w[i] = s.h;
            m.w[i] = s.m;
            l.w[i] = s.l;
        }
    }
};
__device__ __forceinline__ void mma(f4 &acc, const Factor<bf16_bits> &a, const Factor<bf16_bits> &b)
{
    mma(acc, a.f, b.f);
}
__device__ __forceinline__ void mma(f4 &acc, const Factor<float> &a, const Factor<float> &b)
{
    mma(acc, a.m, b.m);
    mma(acc, a.h, b.l);
    mma(acc, a.l, b.h);
    mma(acc, a.h, b.m);
    mma(acc, a.m, b.h);
    mma(acc, a.h, b.h);
}

// A tile of an operand: [SIZE][BK] of rows or [BK][SIZE], in registers on its way to LDS.
template <typename T, bool COLS, int SIZE, int BK> struct Staged {
    static constexpr int WIDTH = COLS ? SIZE : BK, HEIGHT = COLS ? BK : SIZE;
    static constexpr int STRIDE = WIDTH + (COLS ? 32 : 16) / (int)sizeof(T);
    static constexpr int PER_ROW = WIDTH / 8, COUNT = WIDTH * HEIGHT / 8 / 256;
    Raw<T, 8> r[COUNT];

    // rows: how many of them are there from first on; k: likewise
    __device__ __forceinline__ void load(const T *p, int64_t ld, int64_t first, int64_t rows,
                                         int64_t k0, int64_t k)
    {
        const int64_t down = COLS ? k : rows, across = COLS ? rows : k;
        const T *base = p + (COLS ? k0 * ld + first : first * ld + k0);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int at = i * 256 + threadIdx.x, y = at / PER_ROW, x = at % PER_ROW * 8;
            const int64_t left = y < down ? across - x : 0;
            r[i].load(base + (left > 0 ? y * ld + x : 0), left > 8 ? 8 : (int)left);
        }
    }
    __device__ __forceinline__ void put(T *m) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int at = i * 256 + threadIdx.x, y = at / PER_ROW, x = at % PER_ROW * 8;
            T *to = m + y * STRIDE + x;
            if constexpr (sizeof(T) == 2) {
                *(u4 *)to = u4{r[i].w[0], r[i].w[1], r[i].w[2], r[i].w[3]};
            } else {
                *(f4 *)to = f4{r[i].v[0], r[i].v[1], r[i].v[2], r[i].v[3]};
                *(f4 *)(to + 4) = f4{r[i].v[4], r[i].v[5], r[i].v[6], r[i].v[7]};
            }
        }
    }
};

// Four sums of a row of the result, n .. n + 3, through the epilogue.
template <typename T, typename O, int ACT>
__device__ __forceinline__ void finish_as(const ProductArgs &a, int64_t m, int n, f4 v)
{
    const int left = a.N - n;
    if (a.bias) {
        float b[4];
        load_some<4>(a.bias + n, left, b);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] += b[i];
    }
    if (a.pre)
        store4((T *)a.pre + m * a.ld_pre + n, left, v);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = activate<ACT>(v[i]);
    if (a.residual) {
        float r[4];
        load_some<4>((const O *)a.residual + m * a.ld_residual + n, left, r);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] += r[i];
    }
    store4((O *)a.out + m * a.ld_out + n, left, v);
}
template <typename T, int ACT>
__device__ __forceinline__ void finish(const ProductArgs &a, int64_t m, int n, const f4 &v)
{
    if (a.out_bf16) finish_as<T, bf16_bits, ACT>(a, m, n, v);
    else finish_as<T, float, ACT>(a, m, n, v);
}

// A wavefront's results from row m0 and column n0 on, through the epilogue or into the partial sums.
template <typename T, int MT, int NT, int ACT>
__device__ __forceinline__ void finish_tile(const ProductArgs &a, const f4 (&acc)[MT][NT],
                                            int64_t m0, int n0, int64_t split)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int64_t m = m0 + 16 * i + (lane & 15);
            const int n = n0 + 16 * j + 4 * (lane >> 4);
            if (m >= a.M || n >= a.N)
                continue;
            if (a.splits > 1)
                store4(a.partial + (split * a.M + m) * a.N + n, a.N - n, acc[i][j]);
            else
                finish<T, ACT>(a, m, n, acc[i][j]);
        }
}

// Which part of the result a workgroup has.  Workgroups go to the eight XCDs in turn; each gets tiles
// that lie together, whose operands its L2 then holds for all of them.
struct Place {
    int64_t m0, k, k_end;
    int n0, split;
};
template <int BM, int BN> __device__ __forceinline__ Place place(const ProductArgs &a, int64_t first)
{
    const uint32_t across = (uint32_t)(a.N + BN - 1) / BN;
    uint32_t id = blockIdx.x;
    if (gridDim.x % 8 == 0)
        id = id % 8 * (gridDim.x / 8) + id / 8;
    Place x;
    uint32_t column = id % across, row = id / across;
    if (a.splits == 1) {
        // eight rows of tiles at a time, so that what runs at once is a square of them
        const uint32_t rows = gridDim.x / across, group = id / (8 * across);
        const uint32_t high = rows - 8 * group < 8 ? rows - 8 * group : 8;
        const uint32_t in_group = id - group * 8 * across;
        row = 8 * group + in_group % high;
        column = in_group / high;
    }
    x.n0 = (int)column * BN;
    const int64_t rest = first + row;
    if (a.splits > 1) {  // few tiles: in 32 bits
        x.m0 = (int64_t)((uint32_t)rest / (uint32_t)a.splits) * BM;
        x.split = (int)((uint32_t)rest % (uint32_t)a.splits);
    } else {
        x.m0 = rest * BM;
        x.split = 0;
    }
    x.k = x.split * a.split;
    x.k_end = x.k + a.split < a.K ? x.k + a.split : a.K;
    return x;
}

template <typename T, bool A_COLS, bool B_COLS, int BM, int BN, int ACT>
__global__ __launch_bounds__(256, 2) void product_kernel(const ProductArgs a, int64_t first)
{
    constexpr int BK = 128 / (int)sizeof(T);
    using Sa = Staged<T, A_COLS, BM, BK>;
    using Sb = Staged<T, B_COLS, BN, BK>;
    __shared__ __align__(16) T tile_a[2][Sa::HEIGHT * Sa::STRIDE], tile_b[2][Sb::HEIGHT * Sb::STRIDE];
    constexpr int MT = BM / 32, NT = BN / 32;  // 16 x 16 results of a wavefront, a quarter of the tile
    const int wave = threadIdx.x >> 6;
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    const Place x = place<BM, BN>(a, first);
    const int64_t m0 = x.m0, k_first = x.k, k_end = x.k_end;
    const int n0 = x.n0;
    f4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    Sa sa;
    Sb sb;
    auto load = [&](int64_t k) {
        sa.load((const T *)a.a, a.ld_a, m0, a.M - m0, k, k_end - k);
        sb.load((const T *)a.b, a.ld_b, n0, a.N - n0, k, k_end - k);
    };
    load(k_first);
    int at = 0;
    for (int64_t k = k_first; k < k_end; k += BK) {
        sa.put(tile_a[at]);
        sb.put(tile_b[at]);
        __syncthreads();
        if (k + BK < k_end)
            load(k + BK);
#pragma unroll
        for (int kb = 0; kb < BK; kb += 32) {
            Factor<T> fb[NT];
            Frag<T> f;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                operand<T, B_COLS>(f, tile_b[at], Sb::STRIDE, wn + 16 * j, kb);
                fb[j].set(f);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                Factor<T> fa;
                operand<T, A_COLS>(f, tile_a[at], Sa::STRIDE, wm + 16 * i, kb);
                fa.set(f);
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    mma(acc[i][j], fb[j], fa);
            }
        }
        at ^= 1;
    }
    finish_tile<T, MT, NT, ACT>(a, acc, m0 + wm, n0 + wn, x.split);
}

// ---- the product of operands that whole 16-byte pieces hold

// A stage of an operand in LDS is SIZE rows of 128 bytes of k, as lds_off lays them, or as many k of
// SIZE columns, with the groups of 16 columns of a row exchanged, so that what a transposing read
// takes together (bf16: four rows and those eight on; float32: every fourth) lies in different
// banks.
constexpr int kStageRow = 128;
typedef __attribute__((address_space(3))) char lds_char;

template <typename T, int SIZE> struct Columns {
    static constexpr int ROW = SIZE * (int)sizeof(T);  // bytes of a k
    static __device__ __forceinline__ int group(int k)
    {
        if constexpr (sizeof(T) == 4)
            return (k >> 2) & 3;
        else if constexpr (SIZE == 128)
            return (k & 3) | (k >> 1 & 4);
        else
            return (k >> 1 & 1) | (k >> 2 & 2);
    }
};
template <typename T, bool COLS, int SIZE> struct DmaOperand {
    static constexpr int ROW = kStageRow, BK = ROW / (int)sizeof(T), EACH = 16 / (int)sizeof(T);
    static constexpr int LOADS = SIZE * ROW / 4096;  // of 1 KB, by each of four wavefronts
    const char *base;  // the first row, or column, of the next stage
    int64_t step;      // bytes from stage to stage
    int ld, there;     // bytes; rows, or columns, that are there
    int at[LOADS];     // this lane's bytes from the stage's first k
    int piece[LOADS];  // its first k (rows)

    __device__ __forceinline__ DmaOperand(const void *p, int64_t stride, int64_t first, int64_t count,
                                          int64_t k)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        base = (const char *)((const T *)p + (COLS ? k * stride + first : first * stride + k));
        ld = (int)stride * (int)sizeof(T);
        step = COLS ? (int64_t)BK * ld : ROW;
        there = count - first < SIZE ? (int)(count - first) : SIZE;
#pragma unroll
        for (int d = 0; d < LOADS; ++d) {
            const int byte = (wave + 4 * d) * 1024 + lane * 16;
            piece[d] = 0;
            if constexpr (COLS) {
                using L = Columns<T, SIZE>;
                const int k = byte / L::ROW, slot = byte % L::ROW / 16;
                constexpr int PER = (int)sizeof(T);  // pieces of a group: 16 values
                const int col = (slot ^ (L::group(k) * PER)) * EACH;
                at[d] = col < there ? k * ld + col * (int)sizeof(T) : kOutOfRange;
            } else {
                const int line = byte >> 8, slot = byte >> 4 & 15;
                const int q = (slot ^ line) & 7;
                piece[d] = q * EACH;
                at[d] = (2 * line + (slot >> 3)) * ld + q * 16;
            }
        }
    }
    // The next stage, of whose k `left` are there (left > 0).
    __device__ __forceinline__ void issue(uint32_t lds, int64_t left)
    {
        const int n = left < BK ? (int)left : BK;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        // the last row, or k, ends where its last piece does
        const i4 rs = dma_rsrc(base, (uint32_t)(((COLS ? n : there) - 1) * ld +
                                                (COLS ? there : n) * (int)sizeof(T)));
#pragma unroll
        for (int d = 0; d < LOADS; ++d)
            dma_b128(__builtin_amdgcn_readfirstlane(lds + (wave + 4 * d) * 1024), rs,
                     COLS || piece[d] < n ? at[d] : kOutOfRange, 0);
        base += step;
    }
};

// 32 values k from 32 kb on of the 16 rows, or columns, from 16 tile on, of a stage.
template <typename T, bool COLS, int SIZE>
__device__ __forceinline__ void stage_operand(Frag<T> &f, uint32_t stage, int tile, int kb)
{
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    if constexpr (!COLS) {
        if constexpr (sizeof(T) == 2) {
            f.w = *(const u4 *)(lds_char *)(uintptr_t)(stage + tile * 2048 + lds_off(c, 4 * kb + g) * 2);
        } else {
            const f4 a = *(const f4 *)(lds_char *)(uintptr_t)(stage + tile * 2048 + lds_off(c, g) * 2);
            const f4 b = *(const f4 *)(lds_char *)(uintptr_t)(stage + tile * 2048 + lds_off(c, 4 + g) * 2);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                f.v[r] = a[r];
                f.v[4 + r] = b[r];
            }
        }
    } else {
        using L = Columns<T, SIZE>;
        if constexpr (sizeof(T) == 2) {
            const int k = 32 * kb + 8 * g + (c >> 2);
            const uint32_t p = stage + k * L::ROW + (tile ^ L::group(k)) * 32 + (c & 3) * 8;
            typedef __attribute__((address_space(3))) s4 lds_s4;
            const u2 a = __builtin_bit_cast(
                u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(uintptr_t)p));
            const u2 b = __builtin_bit_cast(
                u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(uintptr_t)(p + 4 * L::ROW)));
            f.w = u4{a.x, a.y, b.x, b.y};
        } else {
            const uint32_t p = stage + 4 * g * L::ROW + (tile ^ L::group(4 * g)) * 64 + c * 4;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                f.v[r] = *(const float *)(lds_char *)(uintptr_t)(p + r * L::ROW);
                f.v[4 + r] = *(const float *)(lds_char *)(uintptr_t)(p + (16 + r) * L::ROW);
            }
        }
    }
}

// Eight sums of a row of the result, n .. n + 7, through the epilogue.
template <typename T, typename O, int ACT>
__device__ __forceinline__ void finish_eight(const ProductArgs &a, int64_t m, int n, float (&v)[8])
{
    const int left = a.N - n;
    float r[8];
    if (a.residual)
        load_some<8>((const O *)a.residual + m * a.ld_residual + n, left, r);
    if (a.bias) {
        float b[8];
        load_some<8>(a.bias + n, left, b);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] += b[i];
    }
    if (a.pre)
        store_some<8>((T *)a.pre + m * a.ld_pre + n, left, v);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = activate<ACT>(v[i]);
    if (a.residual)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] += r[i];
    store_some<8>((O *)a.out + m * a.ld_out + n, left, v);
}
// The workgroup's tile through LDS, where the wavefronts' results become whole rows, and out: with
// stores of 8 bytes from where the results are, 16384 x 1536 bf16 results and their z took 34 us
// behind a sum of 64, and 25 so.  A row's 16-byte pieces are exchanged by
// its number, so that 16 rows' pieces of one column lie in different banks.
template <typename T, int BM, int BN, int ACT, int MT, int NT>
__device__ __forceinline__ void finish_rows(const ProductArgs &a, const f4 (&acc)[MT][NT], char *smem,
                                            const Place &at, int wm, int wn)
{
    const int lane = threadIdx.x & 63;
    f4 *tile = (f4 *)smem;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int m = 16 * (wm + i) + (lane & 15), piece = 4 * (wn + j) + (lane >> 4);
            tile[m * (BN / 4) + (piece ^ (m & 15))] = acc[i][j];
        }
    __syncthreads();
    constexpr int PER_ROW = BN / 8;
    const int n = at.n0 + (int)threadIdx.x % PER_ROW * 8;
    if (n >= a.N)
        return;
#pragma unroll 2
    for (int row = threadIdx.x / PER_ROW; row < BM; row += 256 / PER_ROW) {
        const int64_t m = at.m0 + row;
        if (m >= a.M)
            return;
        const int piece = (int)threadIdx.x % PER_ROW * 2;
        const f4 x = tile[row * (BN / 4) + (piece ^ (row & 15))];
        const f4 y = tile[row * (BN / 4) + ((piece + 1) ^ (row & 15))];
        float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        if (a.splits > 1)
            store_some<8>(a.partial + (at.split * a.M + m) * a.N + n, a.N - n, v);
        else if (a.out_bf16)
            finish_eight<T, bf16_bits, ACT>(a, m, n, v);
        else
            finish_eight<T, float, ACT>(a, m, n, v);
    }
}

// Two stages: one on its way while the other is worked on.  (Five of half their depth were slower by a
// fifth: what a step costs besides its loads outweighs their latency.)
template <typename T, bool A_COLS, bool B_COLS, int BM, int BN, int ACT>
__global__ __launch_bounds__(256, 2) void product_dma_kernel(const ProductArgs a, int64_t first)
{
    using Pa = DmaOperand<T, A_COLS, BM>;
    using Pb = DmaOperand<T, B_COLS, BN>;
    constexpr int BK = Pa::BK, A_BYTES = BM * Pa::ROW, STAGE = (BM + BN) * Pa::ROW;
    __shared__ __align__(1024) char smem[2 * STAGE];
    const uint32_t lds = (uint32_t)(uintptr_t)(lds_char *)smem;
    constexpr int MT = BM / 32, NT = BN / 32;  // 16 x 16 results of a wavefront, a quarter of the tile
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave >> 1) * MT, wn = (wave & 1) * NT;
    const Place at = place<BM, BN>(a, first);
    Pa pa(a.a, a.ld_a, at.m0, a.M, at.k);
    Pb pb(a.b, a.ld_b, at.n0, a.N, at.k);
    f4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    uint32_t stage = 0;
    auto issue = [&](int64_t left) {
        pa.issue(lds + stage, left);
        pb.issue(lds + stage + A_BYTES, left);
        stage = STAGE - stage;
    };
    if (at.k < at.k_end)
        issue(at.k_end - at.k);
    for (int64_t left = at.k_end - at.k; left > 0; left -= BK) {
        const uint32_t from = lds + (STAGE - stage);
        phase();
        dma_barrier<0>();  // this stage is there, and the one before it has been read
        phase();
        if (left > BK)
            issue(left - BK);
#pragma unroll
        for (int kb = 0; kb < BK / 32; ++kb) {
            Frag<T> xa[MT], xb[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j)
                stage_operand<T, B_COLS, BN>(xb[j], from + A_BYTES, wn + j, kb);
#pragma unroll
            for (int i = 0; i < MT; ++i)
                stage_operand<T, A_COLS, BM>(xa[i], from, wm + i, kb);
            Factor<T> fb[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j)
                fb[j].set(xb[j]);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                Factor<T> fa;
                fa.set(xa[i]);
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    mma(acc[i][j], fb[j], fa);
            }
        }
        if constexpr (sizeof(T) == 2) {
            // the first half's operands, then the second half's among the first half's products
            constexpr int READS = (A_COLS ? 2 : 1) * MT + (B_COLS ? 2 : 1) * NT, EACH = MT * NT / READS;
            __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
#pragma unroll
            for (int i = 0; i < READS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2 * MT * NT - READS * EACH, 0);
        }
    }
    finish_rows<T, BM, BN, ACT>(a, acc, smem, at, wm, wn);
}

// ---- the product of few rows

// 32 values k from k0 on of row `row`, straight from memory: bf16 8 g .., float32 4 g .. and 16 + 4 g ..
template <typename T, bool PIECES> struct Direct {
    Raw<T, 8> r;
    __device__ __forceinline__ void load(const T *p, int64_t ld, int64_t row, int64_t rows, int k0,
                                         int K)
    {
        const int g = threadIdx.x >> 4 & 3;
        const T *at = p + (row < rows ? row : 0) * ld;
        if constexpr (sizeof(T) == 2) {
            const int k = k0 + 8 * g, left = row < rows ? K - k : 0;
            r.load(at + k, PIECES ? (left > 0 ? 8 : 0) : left);
        } else {
            Raw<T, 4> x, y;
            const int k = k0 + 4 * g, left = row < rows ? K - k : 0;
            x.load(at + k, PIECES ? (left > 0 ? 4 : 0) : left);
            y.load(at + k + 16, PIECES ? (left > 16 ? 4 : 0) : left - 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                r.v[i] = x.v[i];
                r.v[4 + i] = y.v[i];
            }
        }
    }
    __device__ __forceinline__ void factor(Factor<T> &f) const
    {
        Frag<T> x;
        if constexpr (sizeof(T) == 2) {
            x.w = u4{r.w[0], r.w[1], r.w[2], r.w[3]};
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x.v[i] = r.v[i];
        }
        f.set(x);
    }
};

// 16 rows by 16 columns to a workgroup, the sum dealt to eight wavefronts, operands from memory into
// registers with everything of 2048 k in flight (float32: 1024), and one launch.  What a CU has in
// flight from beyond L1 is what bounds it, so the work is spread over many.
template <typename T, bool PIECES, int ACT>
__global__ __launch_bounds__(512) void few_rows_kernel(const ProductArgs a)
{
    __shared__ f4 sums[8][64];
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6;
    const int across = (a.N + 15) / 16, n0 = blockIdx.x % across * 16, K = (int)a.K;
    const int m0 = blockIdx.x / across * 16;
    f4 acc = {0.f, 0.f, 0.f, 0.f};
    // 64 values k to a wavefront at a time, in two steps
    constexpr int DEEP = sizeof(T) == 4 ? 4 : 8, STEP = 8 * 64;
    for (int k0 = wave * 64; k0 < K; k0 += STEP * DEEP / 2) {
        Direct<T, PIECES> w[DEEP], x[DEEP];
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            const int k = k0 + d / 2 * STEP + d % 2 * 32;
            w[d].load((const T *)a.b, a.ld_b, n0 + c16, a.N, k, K);
            x[d].load((const T *)a.a, a.ld_a, m0 + c16, a.M, k, K);
        }
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            Factor<T> fw, fx;
            w[d].factor(fw);
            x[d].factor(fx);
            mma(acc, fw, fx);
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave > 0)
        return;
    f4 v = sums[0][lane];
#pragma unroll
    for (int k = 1; k < 8; ++k)
        v += sums[k][lane];
    const int m = m0 + c16, n = n0 + 4 * g;
    if (m < a.M && n < a.N)
        finish<T, ACT>(a, m, n, v);
}

// The sum of the splits' partial results, in order, through the epilogue.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void join_kernel(const ProductArgs a)
{
    const int64_t per = (a.N + 3) / 4, count = a.M * per, size = a.M * a.N;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < count;
         id += (int64_t)gridDim.x * 256) {
        const int64_t m = id / per;
        const int n = (int)(id % per) * 4;
        const float *p = a.partial + m * a.N + n;
        f4 v = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < a.splits; ++s) {
            float x[4];
            load_some<4>(p + s * size, a.N - n, x);
            v += f4{x[0], x[1], x[2], x[3]};
        }
        finish<T, ACT>(a, m, n, v);
    }
}

// ---- dz
//
// dz goes to memory in the operands' type: with bf16 it is rounded before the two products, as what
// else they multiply is.  Against float64 that takes the gradients' error from 0.0017, which is their
// own rounding, to 0.0023 (16384 x 768 onto 1536, SiLU).  A second bf16 value of what it leaves would
// double the two products' 103 of 140 us and dz's traffic.  The bias's sums take dz as it was.

constexpr int kSlopeWidth = 512;  // columns of a wavefront, eight a lane

template <typename T, typename O, int ACT>
__global__ __launch_bounds__(256) void slope_kernel(const SlopeArgs a, int row_blocks)
{
    __shared__ float sums[4][kSlopeWidth];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = blockIdx.x / row_blocks * kSlopeWidth + lane * 8, left = a.N - n;
    const int64_t block = blockIdx.x % row_blocks;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int64_t step = (int64_t)row_blocks * 4;
#pragma unroll 2
    for (int64_t t = block * 4 + wave; t < a.T; t += step) {
        float d[8];
        load_some<8>((const O *)a.dout + t * a.ld_dout + n, left, d);
        if constexpr (ACT != LBI_ACT_NONE) {
            float z[8];
            load_some<8>((const T *)a.pre + t * a.ld_pre + n, left, z);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                d[i] *= slope<ACT>(z[i]);
        }
        if (a.dz)
            store_some<8>((T *)a.dz + t * a.N + n, left, d);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            sum[i] += d[i];
    }
    if (!a.partial)
        return;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        sums[wave][lane * 8 + i] = sum[i];
    __syncthreads();
    for (int c = threadIdx.x; c < kSlopeWidth; c += 256) {
        const int at = blockIdx.x / row_blocks * kSlopeWidth + c;
        if (at < a.N)
            a.partial[block * a.N + at] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
    }
}

struct ToVector {
    float *out;
    __device__ __forceinline__ void operator()(int64_t c, float v) const { out[c] = v; }
};

template <typename F> hipError_t by_activation(lbi_activation act, F &&f)
{
    if (act == LBI_ACT_SILU) return f(std::integral_constant<int, LBI_ACT_SILU>{});
    if (act == LBI_ACT_GELU) return f(std::integral_constant<int, LBI_ACT_GELU>{});
    return f(std::integral_constant<int, LBI_ACT_NONE>{});
}


// Whether the operands may be loaded straight into LDS: 16-byte pieces of rows that begin and end
// with them, at distances that a buffer's 32 bits hold.
bool in_pieces(const ProductArgs &a)
{
    const int64_t each = a.bf16 ? 8 : 4;
    auto fits = [&](const void *p, int64_t ld, int64_t width) {
        return ((uintptr_t)p & 15) == 0 && ld % each == 0 && width % each == 0 && ld <= 1 << 20;
    };
    return fits(a.a, a.ld_a, a.a_cols ? a.M : a.K) && fits(a.b, a.ld_b, a.b_cols ? a.N : a.K);
}

template <typename T, bool A_COLS, bool B_COLS, int BM, int BN, int ACT>
hipError_t product(const ProductArgs &a, hipStream_t stream)
{
    const int64_t across = (a.N + BN - 1) / BN, down = (a.M + BM - 1) / BM;
    const bool pieces = in_pieces(a);
    return in_launches(down * a.splits, across, [&](int64_t first, dim3 grid) {
        if (pieces)
            product_dma_kernel<T, A_COLS, B_COLS, BM, BN, ACT><<<grid, 256, 0, stream>>>(a, first);
        else
            product_kernel<T, A_COLS, B_COLS, BM, BN, ACT><<<grid, 256, 0, stream>>>(a, first);
    });
}
// Up to 64 rows, no more workgroups than one or two a CU, and a sum that one workgroup goes along
// before two launches would be over: measured with 1 to 64 rows, 64 to 1536 columns and sums of
// 1024 to 16384.  Onto 768 of 1536, bf16: 5.0 us at 64 rows (cut along the sum, in two launches:
// 7.8); onto 64 of 16384 at 16 rows: 30 (14 in two launches); onto 1536 of 4096 at 64: 16 (13).
// One row reads little beside the matrix, and float32's products take two to three times as long.
constexpr int kFewTiles = 384;
bool few_rows(const ProductArgs &a)
{
    if (a.a_cols || a.b_cols || a.M > 64)
        return false;
    const int64_t tiles = (a.M + 15) / 16 * ((a.N + 15) / 16);
    return tiles <= kFewTiles &&
           a.K * (tiles > 256 ? 2 : 1) * (a.M > 1 ? 3 : 2) <= (a.bf16 ? 16000 : 10500);
}
template <typename T, int ACT> hipError_t product_of_few(const ProductArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.M + 15) / 16 * ((a.N + 15) / 16)));
    if (in_pieces(a))
        few_rows_kernel<T, true, ACT><<<grid, 512, 0, stream>>>(a);
    else
        few_rows_kernel<T, false, ACT><<<grid, 512, 0, stream>>>(a);
    return hipGetLastError();
}
template <typename T, bool A_COLS, bool B_COLS, int ACT>
hipError_t product_tiles(const ProductArgs &a, hipStream_t stream)
{
    if constexpr (!A_COLS && !B_COLS)
        if (few_rows(a))
            return product_of_few<T, ACT>(a, stream);
    if (a.tile_m == 64)
        return product<T, A_COLS, B_COLS, 64, 64, ACT>(a, stream);
    if constexpr (sizeof(T) == 2)
        if (a.tile_n == 64)
            return product<T, A_COLS, B_COLS, 128, 64, ACT>(a, stream);
    return product<T, A_COLS, B_COLS, 128, 128, ACT>(a, stream);
}
template <typename T> hipError_t product_by(const ProductArgs &a, hipStream_t stream)
{
    hipError_t e;
    if (a.a_cols)
        e = product_tiles<T, true, true, LBI_ACT_NONE>(a, stream);
    else if (a.b_cols)
        e = product_tiles<T, false, true, LBI_ACT_NONE>(a, stream);
    else
        e = by_activation(a.act, [&](auto act) {
            return product_tiles<T, false, false, decltype(act)::value>(a, stream);
        });
    if (e != hipSuccess || a.splits <= 1)
        return e;
    const int64_t n = (a.M * ((a.N + 3) / 4) + 255) / 256;
    return by_activation(a.act, [&](auto act) {
        join_kernel<T, decltype(act)::value>
            <<<dim3((unsigned)(n < 8192 ? n : 8192)), 256, 0, stream>>>(a);
        return hipGetLastError();
    });
}

}  // namespace

// The tile and the cuts of the sum, from timings of 14 shapes (1 to 16384 rows, sums of 100 to
// 16384) at every tile and 1 to 24 cuts.
//
// The larger a tile, the fewer bytes and (float32) splits a product takes, but two workgroups a CU
// are needed to keep it busy: 128 x 128 from 512 tiles on (float32: 192, its steps being three times
// as long), 128 x 64 from 384 (bf16 alone: fewer than 192 of 128 x 128 never make as many).  bf16,
// 2048 x 2048 x 2048: 31 us with 256 tiles, 27 with 512, 28 with 1024; 16384 x 1536 x 768: 55, 57,
// 66; float32, 4099 x 768 x 1536: 86, 93, 107.
// Fewer tiles than 128 are cut along the sum to about two workgroups a CU, where each keeps at least
// 4 steps (float32: 6) of 20 (24): the second launch costs 3 us and the partial sums' traffic.
// bf16, 512 x 512 x 4096: 34 us whole, 14 in eight; 6707 x 64 x 1104: 10 whole, 11 in two.
int64_t plan_product(ProductArgs &a)
{
    const int64_t unit = a.bf16 ? 64 : 32, steps = (a.K + unit - 1) / unit;
    auto tiles = [&](int m, int n) { return (a.M + m - 1) / m * ((a.N + n - 1) / n); };
    const bool long_sum = steps >= (a.bf16 ? 64 : 128) && tiles(128, 128) >= 32;
    a.tile_m = a.tile_n = 128;
    if (tiles(128, 128) < (a.bf16 ? 512 : 192) && !long_sum) {
        a.tile_n = 64;
        if (!a.bf16 || tiles(128, 64) < 384)
            a.tile_m = 64;
    }
    const int64_t count = tiles(a.tile_m, a.tile_n);
    int64_t splits = 1;
    if (!few_rows(a) && count <= 128 && steps >= (a.bf16 ? 20 : 24)) {
        splits = 512 / count;
        if (splits > steps / (a.bf16 ? 4 : 6)) splits = steps / (a.bf16 ? 4 : 6);
        if (splits > 16) splits = 16;
    }
    const int64_t per = steps > 0 ? (steps + splits - 1) / splits : 1;
    a.split = per * unit;
    a.splits = steps > 0 ? (int32_t)((steps + per - 1) / per) : 1;
    return a.splits > 1 ? a.splits * a.M * a.N : 0;
}

hipError_t launch_product(const ProductArgs &a, hipStream_t stream)
{
    return a.bf16 ? product_by<bf16_bits>(a, stream) : product_by<float>(a, stream);
}

int64_t slope_rows(int64_t T)
{
    const int64_t n = (T + 15) / 16;
    return n < 512 ? n : 512;
}

hipError_t launch_slope(const SlopeArgs &a, float *dbias, hipStream_t stream)
{
    if (a.T > 0) {
        const int blocks = (int)slope_rows(a.T);
        const dim3 grid((unsigned)((a.N + kSlopeWidth - 1) / kSlopeWidth * blocks));
        hipError_t e = by_activation(a.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            if (a.bf16) {
                if (a.out_bf16) slope_kernel<bf16_bits, bf16_bits, ACT><<<grid, 256, 0, stream>>>(a, blocks);
                else slope_kernel<bf16_bits, float, ACT><<<grid, 256, 0, stream>>>(a, blocks);
            } else {
                if (a.out_bf16) slope_kernel<float, bf16_bits, ACT><<<grid, 256, 0, stream>>>(a, blocks);
                else slope_kernel<float, float, ACT><<<grid, 256, 0, stream>>>(a, blocks);
            }
            return hipGetLastError();
        });
        if (e != hipSuccess)
            return e;
    }
    if (!dbias)
        return hipSuccess;
    return sum_rows(a.partial, a.T > 0 ? slope_rows(a.T) : 0, a.N, a.N, ToVector{dbias}, stream);
}

}  // namespace lbi
