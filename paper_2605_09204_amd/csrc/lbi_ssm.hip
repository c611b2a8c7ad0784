// The selective scan: forward over packed sequences, and one token a sequence.
//
// h_t = a_t h_{t-1} + x_t B_t with a_t = exp(D_t A), x_t = D_t u_t, for every
// channel d and state n; y_t = sum_n C_t h_t.  A state and token costs one
// exponential and four float32 operations (exponent, x B, the two
// multiply-adds), N times those of the token's own bytes: at N = 16 the vector
// ALUs bound it, at small N HBM does.
//
// The recurrence is serial in the tokens, and few channels do not fill the GPU.
// Then the tokens are cut into ranges and walked twice (the map of a range is
// h -> exp(A sum D_t) h + its end from zero): once for the ends alone, without C, z
// and y; a small kernel carries the states along the ranges; the second walk
// starts from them and writes y.  The first walk skips all ranges that end with
// their sequence.  Sequences begin and end anywhere in a range.
//
// Measured, 16 states, bf16, gated: 16384 tokens of 1536 channels in 8 sequences
// 202 us (first walk 84, carry 6, second walk 113; the vector ALUs issue in 90 and 95 % of
// the cycles that a CU is busy; walking such sequences once, 192 workgroups, takes
// longer than twice in ranges that fill the GPU); 32768 tokens of one sequence of 768
// channels in float32 214 us (88, 10, 116); one token of 64 sequences, 13.5 MB, 5.7 us.
#include "lbi_ssm.hpp"

namespace lbi {
namespace {

constexpr int kTile = 32;  // tokens staged at a time

// The state with which the sequence of `seg` begins, in a range that ends at t1.
// Where it leaves the range, another workgroup may already have written its new
// state (state_out may be state_in), so the first walk's copy is read.
template <int NS>
__device__ __forceinline__ void begin_states(const Segment &seg, int64_t r, int64_t t1,
                                             uint32_t dn, int nn, float (&h)[NS])
{
    const PassedArgs p = passed();
    const int64_t dN = (int64_t)p->in.D * p->in.N;
    if (!p->in.state_in) {
        zero_states(h);
    } else if (p->cut.joined && seg.end > t1) {
        load_states<NS>(part_of(p->starts + r * dN, dn), nn, h);
    } else {
        const int64_t row = state_row(p->slots, p->n_slots, seg.seq);
        load_states<NS>(part_of(p->in.state_in + (row < 0 ? 0 : row) * dN, dn), row < 0 ? 0 : nn,
                        h);
    }
}

// ENDS: the first walk.  Otherwise the one that writes y and state_out.
template <typename T, int NS, bool ENDS>
__global__ __launch_bounds__(256, NS <= 4 ? 4 : 2) void scan_kernel(const SsmArgs a)
{
    constexpr int NP = 4 * NS, E = NS >= 2 ? NS / 2 : 1;
    constexpr int BROWS = 256 / NP;  // rows of B and C that the workgroup stages at once
    constexpr int UNROLL = NS <= 4 ? 2 : 1;
    __shared__ __align__(16) f2 dx[kTile][kChannels];
    __shared__ __align__(16) float bc[kTile][4][2 * NS];
    __shared__ __align__(16) float ys[ENDS ? 1 : kTile][kPitch];
    const lbi_ssm_inputs &in = a.in;
    const Sequences q = ssm_sequences(in);
    const unsigned row_of = blockIdx.x / (unsigned)a.cut.tiles;
    const int64_t r = row_of + a.cut.first;
    const Tile tile = tile_of(in, (int)(blockIdx.x - row_of * a.cut.tiles));
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4;
    const int c = (tid >> 6) * 16 + (lane & 15);
    const int nn = c < tile.left ? in.N - g * NS : 0;  // states that this lane holds (at most NS)
    const int64_t dN = (int64_t)in.D * in.N;
    const uint32_t dn = (uint32_t)((tile.d0 + c) * in.N + g * NS) * 4u;  // bytes
    int64_t t0, t1;
    range_rows(a.cut, q, r, &t0, &t1);

    if (!ENDS && a.state_out && (in.offsets || in.T == 0)) {
        // empty sequences keep their states
        for (int64_t s = r; s < in.sequences; s += a.cut.ranges) {
            const int64_t row = q.at(s + 1) > q.at(s) ? -1 : state_row(a.slots, a.n_slots, s);
            if (row < 0)
                continue;
            float h[NS];
            load_states<NS>(part_of(in.state_in + (in.state_in ? row * dN : 0), dn), in.state_in ? nn : 0,
                            h);
            store_states<NS>(part_of(a.state_out + row * dN, dn), nn, h);
        }
    }
    if (t0 >= t1)
        return;

    Segment seg;
    float h[NS], total = 0.f;
    int64_t t = t0;
    if constexpr (ENDS) {
        seg.enter(q, t1 - 1, true);
        const bool leaves = seg.end > t1;
        if (tid == 0 && tile.tile == 0 && tile.group == 0)
            a.flags[r] = !leaves || seg.start >= t0 ? kStarts : 0;
        if (!leaves)
            return;  // the next range begins with a sequence of its own
        zero_states(h);
        if (seg.start >= t0) {
            t = seg.start;
            if (in.state_in) {
                const int64_t row = state_row(a.slots, a.n_slots, seg.seq);
                load_states<NS>(part_of(in.state_in + (row < 0 ? 0 : row) * dN, dn), row < 0 ? 0 : nn,
                                h);
                store_states<NS>(part_of(a.starts + r * dN, dn), nn, h);
            }
        }
    } else {
        seg.enter(q, t0, true);
        if (seg.start < t0)
            load_states<NS>(part_of(a.ends + (r - 1) * dN, dn), nn, h);
        else
            begin_states<NS>(seg, r, t1, dn, nn, h);
    }
    float A2[NS];
    load_states<NS>(part_of(in.A, dn), nn, A2);
#pragma unroll
    for (int i = 0; i < NS; ++i)
        A2[i] = power_rate(A2[i]);

    // staging: a row and eight channels a thread, and E values of B and C
    const int row = tid >> 3, ch = (tid & 7) * 8, left = tile.left - ch;
    const int d8 = tile.d0 + ch;
    float bias[8], skip[8];
    load_some<8>(in.delta_bias + (in.delta_bias ? d8 : 0), in.delta_bias ? left : 0, bias);
    load_some<8>(in.skip + (in.skip ? d8 : 0), in.skip && !ENDS ? left : 0, skip);
    Raw<T, 8> ru, rd, rz;
    T rb[E], rc[E];
    const int br = tid / NP, bn = tid % NP, bcol = tile.group * in.N + bn;
    const Plane<T> pu(in.ld_u, row, d8), pd(in.ld_delta, row, d8), pz(in.ld_z, row, d8),
        py(a.ld_y, row, d8), pb(in.ld_B, br, bcol), pc(in.ld_C, br, bcol);
    // The arguments in the loop: read again where 8 and more states a lane leave no scalar
    // registers for them (which went to scratch memory), held where they fit (1 % faster).
    auto arguments = [&]() {
        if constexpr (NS >= 8)
            return passed();
        else
            return &a;
    };
    auto load = [&](int64_t at, int n) {
        const int m = row < n ? left : 0;
        const auto p = arguments();
        ru.load(pu.at(p->in.u, p->in.ld_u, at), m);
        rd.load(pd.at(p->in.delta, p->in.ld_delta, at), m);
        if (!ENDS && p->in.z)
            rz.load(pz.at(p->in.z, p->in.ld_z, at), m);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool there = br + e * BROWS < n && bn < p->in.N;
            rb[e] = there ? *pb.at(p->in.B, p->in.ld_B, at + e * BROWS) : T(0);
            if (!ENDS)
                rc[e] = there ? *pc.at(p->in.C, p->in.ld_C, at + e * BROWS) : T(0);
        }
    };
    auto tile_rows = [&](const Segment &s, int64_t at) {
        const int64_t end = s.end < t1 ? s.end : t1;
        return (int)(end - at < kTile ? end - at : kTile);
    };
    int n = tile_rows(seg, t);
    load(t, n);
    while (true) {
        float u[8];
        Raw<T, 8> z = rz;
        {
            float d[8];
            ru.unpack(u);
            rd.unpack(d);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                d[i] += bias[i];
            steps_of<8>(arguments()->in.softplus, d);
            if (row >= n) {  // rows past the tile's last one change nothing
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    d[i] = u[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                dx[row][ch + i] = f2{d[i], d[i] * u[i]};
            if (NS > 1 || br < kTile) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    bc[br + e * BROWS][bn / NS][bn % NS] = widen(rb[e]);
                    if (!ENDS)
                        bc[br + e * BROWS][bn / NS][NS + bn % NS] = widen(rc[e]);
                }
            }
        }
        __syncthreads();
        const int64_t at = t, upto = t + n;
        const int rows = n;
        const bool ended = upto == seg.end, more = upto < t1;
        const Segment was = seg;
        if (more) {
            if (ended)
                seg.advance(q);
            t = upto;
            n = tile_rows(seg, t);
            load(t, n);
        }
        for (int k0 = 0; k0 < rows; k0 += 4 * UNROLL) {
#pragma unroll
            for (int k = k0; k < k0 + 4 * UNROLL; k += 4) {
                float y[4];
                if (ENDS)  // (in pairs: a long sum keeps more of its digits)
                    total += (dx[k][c].x + dx[k + 1][c].x) + (dx[k + 2][c].x + dx[k + 3][c].x);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f2 p = dx[k + j][c];
                    float b[NS], cc[NS];
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        b[i] = bc[k + j][g][i];
                        if (!ENDS)
                            cc[i] = bc[k + j][g][NS + i];
                    }
                    y[j] = 0.f;
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        h[i] = fmaf(decay(p.x, A2[i]), h[i], p.y * b[i]);
                        if (!ENDS)
                            y[j] = fmaf(cc[i], h[i], y[j]);
                    }
                }
                if (!ENDS)
                    ys[k + g][c] = sum_states(y);
            }
        }
        if (!ENDS && ended) {
            const PassedArgs p = passed();
            if (p->state_out) {
                const int64_t to = state_row(p->slots, p->n_slots, was.seq);
                if (to >= 0)
                    store_states<NS>(part_of(p->state_out + to * p->in.D * p->in.N, dn), nn, h);
            }
            if (more)
                begin_states<NS>(seg, r, t1, dn, nn, h);
        }
        __syncthreads();
        if (!ENDS && row < rows) {
            float y[8], zz[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                y[i] = fmaf(skip[i], u[i], ys[row][ch + i]);
            const auto p = arguments();
            if (p->in.z) {
                z.unpack(zz);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    y[i] *= silu(zz[i]);
            }
            store_some<8>(py.at(p->y, p->ld_y, at), left, y);
        }
        if (!more)
            break;
    }
    if (ENDS) {
        store_states<NS>(part_of(a.ends + r * dN, dn), nn, h);
        if (g == 0 && c < tile.left)
            a.sums[r * in.D + tile.d0 + c] = total;
    }
}

// One token a sequence.  A lane holds four states of a channel, LANES lanes a
// channel; the states are read and written once, 16 bytes a lane, and are
// nearly all of the bytes.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void scan_step_kernel(const SsmArgs a)
{
    constexpr int PER = 256 / LANES;  // channels a workgroup
    const lbi_ssm_inputs &in = a.in;
    const int part = threadIdx.x % LANES, d = (int)blockIdx.x * PER + threadIdx.x / LANES;
    const int n0 = part * 4;
    const bool live = d < in.D;
    const int nn = live ? in.N - n0 : 0, dd = live ? d : 0;
    const int64_t dN = (int64_t)in.D * in.N, dn = (int64_t)dd * in.N + n0;
    float A2[4];
    load_states<4>(in.A + dn, nn, A2);
    const float bias = in.delta_bias ? in.delta_bias[dd] : 0.f;
    const float skip = in.skip ? in.skip[dd] : 0.f;
    const int64_t o = (int64_t)(dd / (in.D / in.G)) * in.N + n0;
    for (int64_t s = blockIdx.y; s < in.sequences; s += gridDim.y) {
        const int64_t row = state_row(a.slots, a.n_slots, s);
        float h[4], b[4], c[4];
        load_states<4>(in.state_in + (row < 0 ? 0 : row * dN + dn), row < 0 ? 0 : nn, h);
        load_some<4>((const T *)in.B + s * in.ld_B + o, nn, b);
        load_some<4>((const T *)in.C + s * in.ld_C + o, nn, c);
        const float u = widen(((const T *)in.u)[s * in.ld_u + dd]);
        float v = widen(((const T *)in.delta)[s * in.ld_delta + dd]) + bias;
        if (in.softplus)
            v = softplus(v);
        const float x = v * u;
        float y = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = fmaf(decay(v, power_rate(A2[i])), h[i], x * b[i]);
            y = fmaf(c[i], h[i], y);
        }
        if (row >= 0)
            store_states<4>(a.state_out + row * dN + dn, nn, h);
        if constexpr (LANES >= 2) y += xchg<1>(y);
        if constexpr (LANES >= 4) y += xchg<2>(y);
        if constexpr (LANES >= 8) y += xchg<7>(y);
        if constexpr (LANES >= 16) y += xchg<8>(y);
        if (live && part == 0) {
            y = fmaf(skip, u, y);
            if (in.z)
                y *= silu(widen(((const T *)in.z)[s * in.ld_z + d]));
            ((T *)a.y)[s * a.ld_y + d] = narrow<T>(y);
        }
    }
}

template <typename T> hipError_t forward(const SsmArgs &a, hipStream_t stream)
{
    return by_states(a.in.N, [&](auto ns) {
        constexpr int NS = decltype(ns)::value;
        if (a.cut.joined) {
            hipError_t e = over_ranges(a, [&](const SsmArgs &b, dim3 grid) {
                scan_kernel<T, NS, true><<<grid, 256, 0, stream>>>(b);
            });
            if (e == hipSuccess)
                e = launch_carry(a, stream);
            if (e != hipSuccess)
                return e;
        }
        return over_ranges(a, [&](const SsmArgs &b, dim3 grid) {
            scan_kernel<T, NS, false><<<grid, 256, 0, stream>>>(b);
        });
    });
}

template <typename T> hipError_t step(const SsmArgs &a, hipStream_t stream)
{
    const int64_t n = a.in.sequences;
    auto run = [&](auto lanes) {
        constexpr int LANES = decltype(lanes)::value;
        const dim3 grid((unsigned)((a.in.D + 256 / LANES - 1) / (256 / LANES)),
                        (unsigned)(n < 65535 ? n : 65535));
        scan_step_kernel<T, LANES><<<grid, 256, 0, stream>>>(a);
        return hipGetLastError();
    };
    if (a.in.N <= 4) return run(std::integral_constant<int, 1>{});
    if (a.in.N <= 8) return run(std::integral_constant<int, 2>{});
    if (a.in.N <= 16) return run(std::integral_constant<int, 4>{});
    if (a.in.N <= 32) return run(std::integral_constant<int, 8>{});
    return run(std::integral_constant<int, 16>{});
}

}  // namespace

// The cut of least cost.  A range's time goes by its tokens, and by how many
// workgroups share its CU: measured on the scan of 16384 tokens, 1536 channels and 16 states
// (192 workgroups to 16 times as many), one of m alike takes 0.4 + 0.55 m of what it takes alone.
// Joined ranges add `again` of that work (the first walk skips one range a
// sequence) and launches worth `launches` tokens; START tokens stand for a
// workgroup's beginning.  Ranges are whole tiles of at least `least` tokens.
SsmCut ssm_cut(int64_t T, int64_t sequences, int32_t D, int32_t G, bool ragged, double again,
               double launches)
{
    constexpr double START = 16;
    constexpr int64_t CUS = 256;
    SsmCut c = {};
    c.tiles = G * ((D / G + kChannels - 1) / kChannels);
    const int64_t rows = ragged || sequences == 0 ? T : T / sequences;
    const int64_t many = ragged || sequences == 0 ? 1 : sequences;
    const int64_t base = many * c.tiles;
    // Sequences of lengths of their own may be short, and a tile holds one
    // sequence: shorter ranges keep the worst case short.
    const int64_t least = ragged ? kTile : 2 * kTile;
    int64_t best = 1, best_tokens = rows;
    double best_cost = 1e300;
    for (int64_t p = 1; p == 1 || (p <= rows / least && base * p <= 16 * CUS);
         p += 1 + p / 8) {
        int64_t tokens = (rows + p - 1) / p;
        tokens = (tokens + kTile - 1) / kTile * kTile;
        const int64_t parts = tokens > 0 ? (rows + tokens - 1) / tokens : 1;
        const double m = (double)((base * parts + CUS - 1) / CUS);
        double cost = ((double)tokens + START) * (0.4 + 0.55 * m);
        if (parts > 1)
            cost = cost * (1.0 + again * (double)(parts - 1) / (double)parts) + launches;
        if (cost < best_cost) {
            best_cost = cost;
            best = parts;
            best_tokens = tokens;
        }
    }
    c.tokens = best_tokens > 0 ? best_tokens : kTile;
    c.per_sequence = ragged ? 0 : (int32_t)best;
    c.ranges = best * many;
    c.joined = best > 1;
    return c;
}

SsmCut ssm_forward_cut(const lbi_ssm_inputs &in, bool ragged)
{
    return ssm_cut(in.T, in.sequences, in.D, in.G, ragged, 0.75, 64);
}

hipError_t launch_ssm_scan(const SsmArgs &a, hipStream_t stream)
{
    return a.in.dt == LBI_BF16 ? forward<bf16_bits>(a, stream) : forward<float>(a, stream);
}

hipError_t launch_ssm_scan_step(const SsmArgs &a, hipStream_t stream)
{
    return a.in.dt == LBI_BF16 ? step<bf16_bits>(a, stream) : step<float>(a, stream);
}

}  // namespace lbi
