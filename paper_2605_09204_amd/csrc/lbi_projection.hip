// Matrix products with bias, activation and residual in their epilogue, and what the gradient of
// one needs beside two more products.
//
//   out = act(x W^T + bias) + residual;   dz = dout act'(z), dx = dz W, dW = dz^T x
//
// The three differ in how the operands lie: the index that is summed runs along the rows of both
// (forward), of one (dx) or of none (dW).  A workgroup takes a BM x BN tile of the result, the
// operands pass through LDS as they lie, and the matrix instructions' operands are read from there
// straight or through the transposing read.
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
    const int across = (a.N + BN - 1) / BN;
    uint32_t id = blockIdx.x;
    // Workgroups go to the eight XCDs in turn; each gets tiles that lie together, whose operands
    // its L2 then holds for all of them.
    if (gridDim.x % 8 == 0)
        id = id % 8 * (gridDim.x / 8) + id / 8;
    const int n0 = (int)(id % across) * BN;
    const int64_t rest = first + id / across;
    const int64_t m0 = rest / a.splits * BM;
    const int64_t k_first = rest % a.splits * a.split;
    const int64_t k_end = k_first + a.split < a.K ? k_first + a.split : a.K;
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
    finish_tile<T, MT, NT, ACT>(a, acc, m0 + wm, n0 + wn, rest % a.splits);
}

// ---- the product of operands that whole 16-byte pieces hold

// A stage of an operand in LDS is SIZE rows (or columns) of 128 bytes of k: rows as lds_off lays
// them, columns as [BK][SIZE] with the 16-value groups of a row exchanged, so that the rows that
// a transposing read takes together (bf16: 4 of them and 4 eight rows on; float32: every fourth)
// lie in different banks.
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
    static constexpr int BK = 128 / (int)sizeof(T), EACH = 16 / (int)sizeof(T);
    static constexpr int LOADS = SIZE / 32;  // of 1 KB, by each of four wavefronts
    const T *base;  // the first row, or column, at k = 0
    int64_t ld;
    int there;      // rows, or columns, that are there
    int at[LOADS];  // this lane's bytes from the stage's first k
    int piece[LOADS];  // its first k (rows) or column

    __device__ __forceinline__ DmaOperand(const void *p, int64_t ld, int64_t first, int64_t count)
        : ld(ld)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        base = (const T *)p + (COLS ? first : first * ld);
        there = count - first < SIZE ? (int)(count - first) : SIZE;
#pragma unroll
        for (int d = 0; d < LOADS; ++d) {
            const int byte = (wave + 4 * d) * 1024 + lane * 16;
            if constexpr (COLS) {
                using L = Columns<T, SIZE>;
                const int k = byte / L::ROW, slot = byte % L::ROW / 16;
                constexpr int PER = (int)sizeof(T);  // pieces of a group: 16 values
                piece[d] = (slot ^ (L::group(k) * PER)) * EACH;
                at[d] = k * (int)ld * (int)sizeof(T) + piece[d] * (int)sizeof(T);
                if (piece[d] >= there)
                    at[d] = kOutOfRange;
            } else {
                const int line = byte >> 8, slot = (byte >> 4 & 15) ^ (line & 7);
                piece[d] = (slot & 7) * EACH;
                at[d] = ((2 * line + (slot >> 3)) * (int)ld + piece[d]) * (int)sizeof(T);
            }
        }
    }
    // the stage from k on, of which `left` are there (left > 0)
    __device__ __forceinline__ void issue(uint32_t lds, int64_t k, int64_t left) const
    {
        const int n = left < BK ? (int)left : BK;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        // the last row, or k, ends where its last piece does
        const int64_t rows = COLS ? n : there, width = COLS ? there : n;
        const i4 rs = dma_rsrc(base + (COLS ? k * ld : k),
                               (uint32_t)(((rows - 1) * ld + width) * (int)sizeof(T)));
#pragma unroll
        for (int d = 0; d < LOADS; ++d) {
            int v = at[d];
            if constexpr (!COLS)
                v = piece[d] < n ? v : kOutOfRange;
            dma_b128(__builtin_amdgcn_readfirstlane(lds + (wave + 4 * d) * 1024), rs, v, 0);
        }
    }
};
typedef __attribute__((address_space(3))) char lds_char;

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

template <typename T, bool A_COLS, bool B_COLS, int BM, int BN, int ACT>
__global__ __launch_bounds__(256, 2) void product_dma_kernel(const ProductArgs a, int64_t first)
{
    constexpr int BK = 128 / (int)sizeof(T), A_BYTES = BM * 128, STAGE = (BM + BN) * 128;
    __shared__ __align__(1024) char smem[2 * STAGE];
    const uint32_t lds = (uint32_t)(uintptr_t)(lds_char *)smem;
    constexpr int MT = BM / 32, NT = BN / 32;  // 16 x 16 results of a wavefront, a quarter of the tile
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave >> 1) * MT, wn = (wave & 1) * NT;
    const int across = (a.N + BN - 1) / BN;
    uint32_t id = blockIdx.x;
    if (gridDim.x % 8 == 0)
        id = id % 8 * (gridDim.x / 8) + id / 8;
    const int n0 = (int)(id % across) * BN;
    const int64_t rest = first + id / across;
    const int64_t m0 = rest / a.splits * BM;
    const int64_t k_first = rest % a.splits * a.split;
    const int64_t k_end = k_first + a.split < a.K ? k_first + a.split : a.K;
    const DmaOperand<T, A_COLS, BM> pa(a.a, a.ld_a, m0, a.M);
    const DmaOperand<T, B_COLS, BN> pb(a.b, a.ld_b, n0, a.N);
    f4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    auto issue = [&](int64_t k, uint32_t stage) {
        pa.issue(stage, k, k_end - k);
        pb.issue(stage + A_BYTES, k, k_end - k);
    };
    if (k_first < k_end)
        issue(k_first, lds);
    uint32_t at = 0;
    for (int64_t k = k_first; k < k_end; k += BK) {
        phase();
        dma_barrier<0>();  // this stage is there, and the one before it has been read
        phase();
        if (k + BK < k_end)
            issue(k + BK, lds + (STAGE - at));
#pragma unroll
        for (int kb = 0; kb < BK / 32; ++kb) {
            Frag<T> xa[MT], xb[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j)
                stage_operand<T, B_COLS, BN>(xb[j], lds + at + A_BYTES, wn + j, kb);
#pragma unroll
            for (int i = 0; i < MT; ++i)
                stage_operand<T, A_COLS, BM>(xa[i], lds + at, wm + i, kb);
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
        at = STAGE - at;
    }
    finish_tile<T, MT, NT, ACT>(a, acc, m0 + 16 * wm, n0 + 16 * wn, rest % a.splits);
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

// The tile: 128 x 128, or 64 x 64 where those would leave CUs without work.
int tile_of(const ProductArgs &a)
{
    const int64_t big = (a.M + 127) / 128 * ((a.N + 127) / 128);
    return big >= 256 || a.K >= 4096 ? 128 : 64;
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

template <typename T, bool A_COLS, bool B_COLS, int TILE, int ACT>
hipError_t product(const ProductArgs &a, hipStream_t stream)
{
    const int64_t across = (a.N + TILE - 1) / TILE, down = (a.M + TILE - 1) / TILE;
    const bool pieces = in_pieces(a);
    return in_launches(down * a.splits, across, [&](int64_t first, dim3 grid) {
        if (pieces)
            product_dma_kernel<T, A_COLS, B_COLS, TILE, TILE, ACT><<<grid, 256, 0, stream>>>(a, first);
        else
            product_kernel<T, A_COLS, B_COLS, TILE, TILE, ACT><<<grid, 256, 0, stream>>>(a, first);
    });
}
template <typename T> hipError_t product_by(const ProductArgs &a, hipStream_t stream)
{
    const bool big = tile_of(a) == 128;
    hipError_t e;
    if (a.a_cols)
        e = big ? product<T, true, true, 128, LBI_ACT_NONE>(a, stream)
                : product<T, true, true, 64, LBI_ACT_NONE>(a, stream);
    else if (a.b_cols)
        e = big ? product<T, false, true, 128, LBI_ACT_NONE>(a, stream)
                : product<T, false, true, 64, LBI_ACT_NONE>(a, stream);
    else
        e = by_activation(a.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            return big ? product<T, false, false, 128, ACT>(a, stream)
                       : product<T, false, false, 64, ACT>(a, stream);
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

int64_t plan_product(ProductArgs &a)
{
    const int tile = tile_of(a);
    const int64_t tiles = (a.M + tile - 1) / tile * ((a.N + tile - 1) / tile);
    const int64_t unit = a.bf16 ? 64 : 32;
    const int64_t steps = (a.K + unit - 1) / unit;
    // two workgroups a CU, and at least eight steps each
    int64_t splits = 512 / tiles;
    if (splits > steps / 8) splits = steps / 8;
    if (splits < 1) splits = 1;
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
