// Gradient of the selective scan, from the forward's inputs alone.
//
// With g_t the gradient of h_t, walking back from g = that of the final state:
//     g += e_t C_t            (e_t = dy_t silu(z_t))
//     dC_t = sum_d e_t h_t,   dB_t = sum_d g x_t,   dx_t = sum_n g B_t
//     q = a_t g h_{t-1},      dD_t = u_t dx_t + sum_n q A,   dA = sum_t q D_t
//     g <- a_t g
// The walk back needs h_t, which the decays do not allow to be undone, so the
// tokens are walked twice.  The first walk goes forward and leaves a mark (the
// state) every STEP tokens in memory.  The second goes back, STEP tokens at a
// time: from the mark it forms their states again, keeps them in registers with
// their decays, and takes the gradients from them.  So a state and token costs
// two exponentials and about 20 float32 operations in all, and the marks N / STEP
// float32 values a channel and token: the vector ALUs bound it.
//
// Where the tokens are cut into ranges (as in the forward scan), the first walk
// starts every range from zeros and also sums what its tokens send to the
// gradient at its start; two small kernels carry states forward and gradients
// back along the ranges; a mark is then completed by the state at its range's
// start, times the decay up to the mark.
//
// dB and dC are sums over the channels: over the 16 lanes of a row by exchanges
// that halve the values at each stage, over wavefronts in LDS, over workgroups
// as partial sums in memory, added by a last kernel in a fixed order.  So are
// the sums over tokens (dA, dskip, ddelta_bias), range by range.
//
// Measured, 16 states, bf16, gated, 16384 tokens of 1536 channels in 8 sequences:
// 555 us (first walk 152, carry 8, second walk 380, sums of dB and dC 10, of the
// parameters 5; the vector ALUs issue in 93 % of the first walk's and 83 % of the second's
// busy cycles, and the second's last workgroups leave a sixth of the CUs idle at its end).
#include "lbi_ssm.hpp"

namespace lbi {
namespace {

// Tokens between marks, and whether their decays stay in registers too.
constexpr int step_of(int NS) { return NS <= 8 ? 8 : 4; }
constexpr bool keeps_decays(int NS) { return NS <= 4; }
constexpr int kSweep = 32;  // tokens that the first walk stages at a time

// The first walk.  JOINED: ranges are entered in their middle.
template <typename T, int NS, bool JOINED>
__global__ __launch_bounds__(256, NS <= 2 ? 4 : (NS == 4 ? 3 : (NS == 8 ? 2 : 1))) void sweep_kernel(const SsmArgs a)
{
    constexpr int NP = 4 * NS, E = NS >= 2 ? NS / 2 : 1, STEP = step_of(NS);
    constexpr int BROWS = 256 / NP;  // rows of B and C that the workgroup stages at once
    __shared__ __align__(16) f2 dx[kSweep][kChannels];
    __shared__ __align__(16) float bc[kSweep][4][2 * NS];
    __shared__ float es[JOINED ? kSweep : 1][kChannels];
    const lbi_ssm_inputs &in = a.in;
    const Sequences q = ssm_sequences(in);
    const unsigned row_of = blockIdx.x / (unsigned)a.cut.tiles;
    const int64_t r = row_of + a.cut.first;
    const Tile tile = tile_of(in, (int)(blockIdx.x - row_of * a.cut.tiles));
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4;
    const int c = (tid >> 6) * 16 + (lane & 15);
    const int nn = c < tile.left ? in.N - g * NS : 0;
    const int64_t dN = (int64_t)in.D * in.N;
    const uint32_t dn = (uint32_t)((tile.d0 + c) * in.N + g * NS) * 4u;  // bytes
    int64_t t0, t1;
    range_rows(a.cut, q, r, &t0, &t1);
    if (t0 >= t1)
        return;
    Segment seg;
    seg.enter(q, t0, true);
    const bool entered = JOINED && seg.start < t0;  // by a sequence under way
    const bool through = entered && seg.end > t1;   // which also leaves it
    bool first = entered;                           // still in that sequence
    float h[NS], A2[NS], total = 0.f;
    zero_states(h);
    auto begin = [&]() {
        if (in.state_in)
            load_states<NS>(part_of(in.state_in + seg.seq * dN, dn), nn, h);
        else
            zero_states(h);
    };
    if (!entered)
        begin();
    load_states<NS>(part_of(in.A, dn), nn, A2);
#pragma unroll
    for (int i = 0; i < NS; ++i)
        A2[i] = power_rate(A2[i]);
    // what the first sequence's tokens send to the gradient at the range's start
    float head[NS], way[NS];  // way: the decay from the start
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        head[i] = 0.f;
        way[i] = 1.f;
    }

    const int row = tid >> 3, ch = (tid & 7) * 8, left = tile.left - ch;
    const int d8 = tile.d0 + ch;
    float bias[8];
    load_some<8>(in.delta_bias + (in.delta_bias ? d8 : 0), in.delta_bias ? left : 0, bias);
    Raw<T, 8> ru, rd, rz, re;
    T rb[E], rc[E];
    const int br = tid / NP, bn = tid % NP, bcol = tile.group * in.N + bn;
    const Plane<T> pu(in.ld_u, row, d8), pd(in.ld_delta, row, d8), pz(in.ld_z, row, d8),
        pe(a.ld_dy, row, d8), pb(in.ld_B, br, bcol), pc(in.ld_C, br, bcol);
    auto load = [&](int64_t at, int n, bool heads) {
        const int m = row < n ? left : 0;
        const SsmArgs *const p = &a;
        ru.load(pu.at(p->in.u, p->in.ld_u, at), m);
        rd.load(pd.at(p->in.delta, p->in.ld_delta, at), m);
        if (JOINED && heads) {
            re.load(pe.at(p->dy, p->ld_dy, at), m);
            if (p->in.z)
                rz.load(pz.at(p->in.z, p->in.ld_z, at), m);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool there = br + e * BROWS < n && bn < p->in.N;
            rb[e] = there ? *pb.at(p->in.B, p->in.ld_B, at + e * BROWS) : T(0);
            if (JOINED && heads)
                rc[e] = there ? *pc.at(p->in.C, p->in.ld_C, at + e * BROWS) : T(0);
        }
    };
    auto tile_rows = [&](int64_t at) {
        const int64_t end = seg.end < t1 ? seg.end : t1;
        return (int)(end - at < kSweep ? end - at : kSweep);
    };
    int64_t t = t0, from = t0;  // from: where marks of this sequence are counted from
    int n = tile_rows(t);
    load(t, n, first);
    while (true) {
        {
            float u[8], d[8];
            ru.unpack(u);
            rd.unpack(d);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                d[i] += bias[i];
            steps_of<8>(in.softplus, d);
            if (row >= n) {  // rows past the tile's last one change nothing
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    d[i] = u[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                dx[row][ch + i] = f2{d[i], d[i] * u[i]};
            if (JOINED && first) {
                float e[8], z[8];
                re.unpack(e);
                if (in.z) {
                    rz.unpack(z);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        e[i] *= silu(z[i]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    es[row][ch + i] = e[i];
            }
            if (NS > 1 || br < kSweep) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    bc[br + e * BROWS][bn / NS][bn % NS] = widen(rb[e]);
                    if (JOINED && first)
                        bc[br + e * BROWS][bn / NS][NS + bn % NS] = widen(rc[e]);
                }
            }
        }
        __syncthreads();
        const int64_t at = t, upto = t + n;
        const int rows = n;
        const bool ended = upto == seg.end, more = upto < t1;
        const bool heads = first;
        const int64_t seq = seg.seq, begun = from;
        const bool open = entered && from == t0;  // the sequence came from the range before
        if (more) {
            if (ended) {
                seg.advance(q);
                first = false;
                from = upto;
            }
            t = upto;
            n = tile_rows(t);
            load(t, n, first);
        }
        for (int k = 0; k < rows; k += 4) {
            if ((k % STEP) == 0 && at + k > begun) {
                const int64_t m = (at + k) / STEP;
                store_states<NS>(part_of(a.marks + m * dN, dn), nn, h);
                if (JOINED && open && g == 0 && c < tile.left)
                    a.mark_sums[m * in.D + tile.d0 + c] = total;
            }
            if (JOINED)  // (in pairs: a long sum keeps more of its digits)
                total += (dx[k][c].x + dx[k + 1][c].x) + (dx[k + 2][c].x + dx[k + 3][c].x);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f2 p = dx[k + j][c];
                float b[NS], w[NS];
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    b[i] = bc[k + j][g][i];
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    w[i] = decay(p.x, A2[i]);
                    h[i] = fmaf(w[i], h[i], p.y * b[i]);
                }
                if (JOINED && heads) {
                    const float e = es[k + j][c];
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        way[i] *= w[i];
                        head[i] = fmaf(way[i], e * bc[k + j][g][NS + i], head[i]);
                    }
                }
            }
        }
        if (JOINED && ended && heads && a.dstate_out) {
            float e[NS];
            load_states<NS>(part_of(a.dstate_out + seq * dN, dn), nn, e);
#pragma unroll
            for (int i = 0; i < NS; ++i)
                head[i] = fmaf(way[i], e[i], head[i]);
        }
        if (ended && more) {
            total = 0.f;
            begin();
        }
        __syncthreads();
        if (!more)
            break;
    }
    if (JOINED) {
        // a range that no sequence enters sends no gradient back, one that none
        // leaves no state on: what is stored then is not used
        store_states<NS>(part_of(a.ends + r * dN, dn), nn, h);
        store_states<NS>(part_of(a.heads + r * dN, dn), nn, head);
        if (g == 0 && c < tile.left)
            a.sums[r * in.D + tile.d0 + c] = total;
        if (tid == 0 && tile.tile == 0 && tile.group == 0)
            a.flags[r] = through ? 0 : (kStarts | kEnds);
    }
}

// The second walk.  Wavefronts a SIMD: as many as its registers allow.
template <typename T> constexpr int waves_of(int NS)
{
    return NS <= 4 && sizeof(T) == 2 ? 3 : (NS <= 8 ? 2 : 1);
}
template <typename T, int NS, bool JOINED>
__global__ __launch_bounds__(256, waves_of<T>(NS)) void gradient_kernel(const SsmArgs a)
{
    constexpr int STEP = step_of(NS), NP = 4 * NS;
    constexpr int V = 2;                             // channels a thread stages
    constexpr int E = (STEP * NP + 255) / 256;       // B (and C) values a thread stages
    constexpr int BROWS = 256 / NP;                  // rows of them staged at once
    constexpr int PER = NS <= 2 ? 4 : (NS == 4 ? 2 : 1);  // tokens whose dB, dC are summed at once
    constexpr int LIVE = PER * NS * 2;               // their values in a lane: 16, or 8 and 32 at the ends
    constexpr bool KEEP = keeps_decays(NS);
    constexpr int LANES_V = kChannels / V;           // threads a row
    __shared__ __align__(16) f2 dx[STEP][kChannels];
    __shared__ float es[STEP][kChannels];
    __shared__ __align__(16) float bc[STEP][4][2 * NS];
    __shared__ __align__(16) float ob[STEP][kPitch], oa[STEP][kPitch], oy[STEP][kPitch];
    __shared__ __align__(16) float red[4][STEP][NP][2];
    // per channel: delta_bias and skip; and each staging thread's share of the
    // sums for dskip and ddelta_bias
    __shared__ __align__(16) float par[2][kChannels], sums[2][256 / LANES_V][kChannels];
    const lbi_ssm_inputs &in = a.in;
    const Sequences q = ssm_sequences(in);
    const unsigned row_of = blockIdx.x / (unsigned)a.cut.tiles;
    const int64_t r = row_of + a.cut.first;
    const Tile tile = tile_of(in, (int)(blockIdx.x - row_of * a.cut.tiles));
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, wave = tid >> 6;
    const int c = wave * 16 + (lane & 15);
    const int nn = c < tile.left ? in.N - g * NS : 0;
    const int64_t dN = (int64_t)in.D * in.N;
    const uint32_t dn = (uint32_t)((tile.d0 + c) * in.N + g * NS) * 4u;  // bytes
    int64_t t0, t1;
    range_rows(a.cut, q, r, &t0, &t1);
    if (a.out.dstate_in && (in.offsets || in.T == 0)) {
        // the states of empty sequences pass through
        for (int64_t s = r; s < in.sequences; s += a.cut.ranges) {
            if (q.at(s + 1) > q.at(s))
                continue;
            float e[NS];
            load_states<NS>(part_of(a.dstate_out + (a.dstate_out ? s * dN : 0), dn),
                            a.dstate_out ? nn : 0, e);
            store_states<NS>(part_of(a.out.dstate_in + s * dN, dn), nn, e);
        }
    }
    if (t0 >= t1)
        return;  // only without tokens at all, when the sums have no rows
    float A2[NS], dA[NS], gr[NS], hs[STEP + 1][NS];
    load_states<NS>(part_of(in.A, dn), nn, A2);
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        A2[i] = power_rate(A2[i]);
        dA[i] = 0.f;
    }

    const int row = tid / LANES_V, ch = (tid % LANES_V) * V, left = tile.left - ch;
    const int dv = tile.d0 + ch;
    if (tid < kChannels) {
        par[0][tid] = in.delta_bias && tid < tile.left ? in.delta_bias[tile.d0 + tid] : 0.f;
        par[1][tid] = in.skip && tid < tile.left ? in.skip[tile.d0 + tid] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        sums[0][row][ch + i] = sums[1][row][ch + i] = 0.f;
    __syncthreads();
    Raw<T, V> ru, rd, rz, re;
    T rb[E], rc[E];
    const int br = tid / NP, bn = tid % NP, bcol = tile.group * in.N + bn;
    const Plane<T> pu(in.ld_u, row, dv), pd(in.ld_delta, row, dv), pz(in.ld_z, row, dv),
        pe(a.ld_dy, row, dv), pb(in.ld_B, br, bcol), pc(in.ld_C, br, bcol);
    auto load = [&](int64_t at, int n) {
        const int m = row < n ? left : 0;
        const PassedArgs p = passed();
        ru.load(pu.at(p->in.u, p->in.ld_u, at), m);
        rd.load(pd.at(p->in.delta, p->in.ld_delta, at), m);
        re.load(pe.at(p->dy, p->ld_dy, at), m);
        if (p->in.z)
            rz.load(pz.at(p->in.z, p->in.ld_z, at), m);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool there = br + e * BROWS < n && bn < p->in.N;
            rb[e] = there ? *pb.at(p->in.B, p->in.ld_B, at + e * BROWS) : T(0);
            rc[e] = there ? *pc.at(p->in.C, p->in.ld_C, at + e * BROWS) : T(0);
        }
    };
    // The piece of a sequence within the range, rows lo .. hi - 1, and in it the
    // steps from the last one back.
    Segment seg;
    int64_t lo, t;
    int n;
    auto enter = [&](int64_t last) {
        seg.enter(q, last, true);
        lo = seg.start > t0 ? seg.start : t0;
        const int64_t hi = seg.end < t1 ? seg.end : t1;
        t = lo + (hi - 1 - lo) / STEP * STEP;
        n = (int)(hi - t);
    };
    auto begin = [&](bool leaves) {
        const PassedArgs p = passed();
        const int64_t dN = (int64_t)p->in.D * p->in.N;
        if (JOINED && leaves)
            load_states<NS>(part_of(p->heads + (r + 1) * dN, dn), nn, gr);
        else
            load_states<NS>(part_of(p->dstate_out + (p->dstate_out ? seg.seq * dN : 0), dn),
                            p->dstate_out ? nn : 0, gr);
    };
    // The state before the step at t, loaded ahead of its use: the piece's first
    // state, or a mark, which is completed by the state that entered the range.
    float next_h[NS], next_sum = 0.f, entry[NS];
    bool has_entry = false;
    zero_states(entry);
    auto load_state = [&]() {
        const PassedArgs p = passed();
        const int64_t dN = (int64_t)p->in.D * p->in.N;
        if (JOINED && seg.start < t0 && !has_entry) {
            load_states<NS>(part_of(p->ends + (r - 1) * dN, dn), nn, entry);
            has_entry = true;
        }
        if (t > lo) {
            const int64_t m = t / STEP;
            load_states<NS>(part_of(p->marks + m * dN, dn), nn, next_h);
            if (JOINED && seg.start < t0)
                next_sum = c < tile.left ? p->mark_sums[m * p->in.D + tile.d0 + c] : 0.f;
        } else if (JOINED && seg.start < t0) {
#pragma unroll
            for (int i = 0; i < NS; ++i)
                next_h[i] = entry[i];
        } else if (p->in.state_in) {
            load_states<NS>(part_of(p->in.state_in + seg.seq * dN, dn), nn, next_h);
        } else {
            zero_states(next_h);
        }
    };
    enter(t1 - 1);
    begin(seg.end > t1);
    load(t, n);
    load_state();
    while (true) {
        const Raw<T, V> was_u = ru, was_d = rd, was_e = re, was_z = rz;
        {
            float u[V], d[V], e[V], z[V];
            ru.unpack(u);
            rd.unpack(d);
            re.unpack(e);
            if (in.z)
                rz.unpack(z);
#pragma unroll
            for (int i = 0; i < V; ++i)
                d[i] += par[0][ch + i];
            steps_of<V>(in.softplus, d);
            if (row >= n) {  // rows past the step's last one change nothing
#pragma unroll
                for (int i = 0; i < V; ++i)
                    d[i] = u[i] = 0.f;
            }
            if (in.z) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    e[i] *= silu(z[i]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (LANES_V * STEP >= 256 || row < STEP) {
                    dx[row][ch + i] = f2{d[i], d[i] * u[i]};
                    es[row][ch + i] = e[i];
                }
            }
            if (STEP * NP % 256 == 0 || br < STEP) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    bc[br + e * BROWS][bn / NS][bn % NS] = widen(rb[e]);
                    bc[br + e * BROWS][bn / NS][NS + bn % NS] = widen(rc[e]);
                }
            }
        }
        // the state before the step
#pragma unroll
        for (int i = 0; i < NS; ++i)
            hs[0][i] = next_h[i];
        if (JOINED && seg.start < t0 && t > lo) {
            bool far = false;  // a state of the wavefront grows by 2^127
#pragma unroll
            for (int i = 0; i < NS; ++i)
                far |= A2[i] * next_sum > 126.f;
            if (__ballot(far)) {
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    hs[0][i] += grown(entry[i], A2[i] * next_sum);
            } else {
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    hs[0][i] = fmaf(__builtin_amdgcn_exp2f(A2[i] * next_sum), entry[i], hs[0][i]);
            }
        }
        __syncthreads();
        const int64_t at = t, from = lo, seq = seg.seq;
        const int rows = n;
        const bool whole = lo == seg.start;       // the piece begins with its sequence
        const bool piece = t == lo, more = t > t0;  // the piece's last step; rows remain
        if (more) {
            if (piece) {
                enter(from - 1);
            } else {
                t -= STEP;
                n = STEP;
            }
            load(t, n);
            load_state();
        }
        float w[KEEP ? STEP : 1][NS];
#pragma unroll
        for (int k = 0; k < STEP; ++k) {
            const f2 p = dx[k][c];
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const float v = decay(p.x, A2[i]);
                if constexpr (KEEP)
                    w[k][i] = v;
                hs[k + 1][i] = fmaf(v, hs[k][i], p.y * bc[k][g][i]);
            }
        }
        float part[NS];  // the step's share of dA
        zero_states(part);
#pragma unroll
        for (int k = STEP - 4; k >= 0; k -= 4) {
            // indexes that the compiler cannot tell from other ones, so that dx and bc
            // are read again from LDS: what the way forward has read would
            // otherwise be kept in registers, and spill
            int c2 = c, g2 = g;
            asm volatile("" : "+v"(c2), "+v"(g2));
            __builtin_amdgcn_sched_barrier(0);
            float sb[4], sa[4], sy[4];
#pragma unroll
            for (int p0 = 4 - PER; p0 >= 0; p0 -= PER) {
                __builtin_amdgcn_sched_barrier(0);
                float v[LIVE];
#pragma unroll
                for (int p = PER - 1; p >= 0; --p) {
                    const int j = p0 + p, kk = k + j;
                    const f2 x = dx[kk][c2];
                    const float e = es[kk][c2];
                    float bcs[2 * NS];
                    read_lds<2 * NS>(bc[kk][g2], bcs);
                    sb[j] = sa[j] = sy[j] = 0.f;
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        const float b = bcs[i], cc = bcs[NS + i];
                        float dec;
                        if constexpr (KEEP) dec = w[kk][i];
                        else dec = decay(x.x, A2[i]);
                        gr[i] = fmaf(e, cc, gr[i]);
                        sy[j] = fmaf(cc, hs[kk + 1][i], sy[j]);
                        sb[j] = fmaf(gr[i], b, sb[j]);
                        v[(p * NS + i) * 2] = gr[i] * x.y;
                        v[(p * NS + i) * 2 + 1] = e * hs[kk + 1][i];
                        gr[i] *= dec;
                        const float qq = gr[i] * hs[kk][i];
                        sa[j] = fmaf(qq, A2[i], sa[j]);
                        part[i] = fmaf(qq, x.x, part[i]);
                        pin(part[i]);
                    }
                    pin(sy[j]);
                }
                // over the 16 channels of the lane row
                group_reduce<16, LIVE>(v, lane & 15);
                constexpr int HOLD = LIVE / 16 > 0 ? LIVE / 16 : 1;  // values a lane ends with
                constexpr int SHIFT = LIVE >= 16 ? 0 : ilog2(16 / LIVE);
                const int at0 = ((lane & 15) >> SHIFT) * HOLD;
                if ((lane & ((1 << SHIFT) - 1)) == 0)
#pragma unroll
                    for (int x = 0; x < HOLD; ++x) {
                        const int o = at0 + x;
                        red[wave][k + p0 + o / (2 * NS)][g * NS + o / 2 % NS][o % 2] = v[x];
                    }
            }
            ob[k + g][c] = sum_states(sb);
            oa[k + g][c] = sum_states(sa);
            if (in.z)
                oy[k + g][c] = sum_states(sy);
        }
#pragma unroll
        for (int i = 0; i < NS; ++i)
            dA[i] += part[i];
        if (piece) {
            const PassedArgs p = passed();
            if (whole && p->out.dstate_in)
                store_states<NS>(part_of(p->out.dstate_in + seq * p->in.D * p->in.N, dn), nn, gr);
            if (more)
                begin(false);
        }
        __syncthreads();
        if (row < rows) {
            float u[V], raw[V], du[V], dd[V];
            was_u.unpack(u);
            was_d.unpack(raw);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float sx = ob[row][ch + i], e = es[row][ch + i];
                du[i] = fmaf(sx, dx[row][ch + i].x, par[1][ch + i] * e);
                dd[i] = fmaf(oa[row][ch + i], kLn2, sx * u[i]);
                if (in.softplus)
                    dd[i] *= sigmoid(raw[i] + par[0][ch + i]);
                sums[0][row][ch + i] = fmaf(e, u[i], sums[0][row][ch + i]);
                sums[1][row][ch + i] += dd[i];
            }
            const PassedArgs p = passed();
            store_some<V>(Plane<T>(p->out.ld_du, row, dv).at(p->out.du, p->out.ld_du, at), left, du);
            store_some<V>(Plane<T>(p->out.ld_ddelta, row, dv)
                             .at(p->out.ddelta, p->out.ld_ddelta, at), left, dd);
            if (in.z) {
                float e0[V], z[V], dz[V];
                was_e.unpack(e0);
                was_z.unpack(z);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float y = fmaf(par[1][ch + i], u[i], oy[row][ch + i]);
                    dz[i] = e0[i] * y * silu_slope(z[i], sigmoid(z[i]));
                }
                store_some<V>(Plane<T>(p->out.ld_dz, row, dv).at(p->out.dz, p->out.ld_dz, at), left,
                             dz);
            }
        }
        for (int i = tid; i < STEP * NP; i += 256) {
            const PassedArgs p = passed();
            const int br = i / NP, bn = i % NP;
            if (br < rows && bn < p->in.N) {
                f2 s = *(const f2 *)red[0][br][bn];
#pragma unroll
                for (int x = 1; x < 4; ++x) {
                    const f2 o = *(const f2 *)red[x][br][bn];
                    s.x += o.x;
                    s.y += o.y;
                }
                const int64_t row0 = (int64_t)tile.tile * p->in.T + at, gn = p->in.G * p->in.N;
                *(f2 *)lane_address(p->part_bc + row0 * gn * 2,
                                    (uint32_t)(br * (int)gn + tile.group * p->in.N + bn) * 8u) = s;
            }
        }
        if (!more)
            break;
        // No barrier: what the threads write before the next one are entries of
        // dx and es that only they themselves read here, and bc, that none does.
    }
    float *par_row = a.part_par + r * (dN + 2 * in.D);
    store_states<NS>(part_of(par_row, dn), nn, dA);
    __syncthreads();
    if (tid < 2 * kChannels && tid % kChannels < tile.left) {
        const int which = tid / kChannels, at = tid % kChannels;
        float v = 0.f;
#pragma unroll
        for (int x = 0; x < 256 / LANES_V; ++x)
            v += sums[which][x][at];
        par_row[dN + which * in.D + tile.d0 + at] = v;
    }
}

struct ToParameters {
    float *dA, *dskip, *dbias;
    int64_t dN;
    int32_t D;
    __device__ __forceinline__ void operator()(int64_t c, float v) const
    {
        if (c < dN) {
            dA[c] = v;
        } else if (c < dN + D) {
            if (dskip)
                dskip[c - dN] = v;
        } else if (dbias) {
            dbias[c - dN - D] = v;
        }
    }
};

// dB and dC from the channel tiles' sums, two float2 a thread and tile.
template <typename T> __global__ __launch_bounds__(256) void sum_tiles_kernel(const SsmArgs a, int64_t first)
{
    const int64_t gn = (int64_t)a.in.G * a.in.N, all = a.in.T * gn;
    const int64_t i = (first + blockIdx.x) * 256 + threadIdx.x;
    if (i >= all)
        return;
    const int tiles = a.cut.tiles / a.in.G;
    const f2 *p = (const f2 *)a.part_bc + i;
    f2 s = {0.f, 0.f};
    int k = 0;
    for (; k + 8 <= tiles; k += 8) {
        f2 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = p[(k + j) * all];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s.x += v[j].x;
            s.y += v[j].y;
        }
    }
    for (; k < tiles; ++k) {
        const f2 v = p[k * all];
        s.x += v.x;
        s.y += v.y;
    }
    const int64_t t = i / gn, o = i - t * gn;
    ((T *)a.out.dB)[t * a.out.ld_dB + o] = narrow<T>(s.x);
    ((T *)a.out.dC)[t * a.out.ld_dC + o] = narrow<T>(s.y);
}

template <typename T, int NS, bool JOINED> hipError_t walks(const SsmArgs &a, hipStream_t stream)
{
    hipError_t e = hipSuccess;
    // without ranges to join, marks are needed only past a sequence's first step
    if (JOINED || a.in.offsets || a.in.T / a.in.sequences > step_of(NS))
        e = over_ranges(a, [&](const SsmArgs &b, dim3 grid) {
            sweep_kernel<T, NS, JOINED><<<grid, 256, 0, stream>>>(b);
        });
    if (JOINED && e == hipSuccess)
        e = launch_carry(a, stream);
    if (e != hipSuccess)
        return e;
    return over_ranges(a, [&](const SsmArgs &b, dim3 grid) {
        gradient_kernel<T, NS, JOINED><<<grid, 256, 0, stream>>>(b);
    });
}

template <typename T> hipError_t backward(const SsmArgs &a, hipStream_t stream)
{
    hipError_t e = hipSuccess;
    if (a.in.sequences > 0)
        e = by_states(a.in.N, [&](auto ns) {
            constexpr int NS = decltype(ns)::value;
            return a.cut.joined ? walks<T, NS, true>(a, stream) : walks<T, NS, false>(a, stream);
        });
    if (e != hipSuccess)
        return e;
    const int64_t values = a.in.T * a.in.G * a.in.N;
    if (values > 0) {
        e = in_launches((values + 255) / 256, 1, [&](int64_t first, dim3 grid) {
            sum_tiles_kernel<T><<<grid, 256, 0, stream>>>(a, first);
        });
        if (e != hipSuccess)
            return e;
    }
    const int64_t dN = (int64_t)a.in.D * a.in.N, cols = dN + 2 * a.in.D;
    return sum_rows(a.part_par, a.in.T > 0 ? a.cut.ranges : 0, cols, cols,
                    ToParameters{a.out.dA, a.out.dskip, a.out.ddelta_bias, dN, a.in.D}, stream);
}

}  // namespace

// Joined ranges cost the first walk its sums for the gradients at their starts.
SsmCut ssm_backward_cut(const lbi_ssm_inputs &in, bool ragged)
{
    return ssm_cut(in.T, in.sequences, in.D, in.G, ragged, 0.15, 16);
}

int32_t ssm_backward_step(int32_t N) { return N <= 32 ? step_of(8) : step_of(16); }

hipError_t launch_ssm_scan_backward(const SsmArgs &a, hipStream_t stream)
{
    return a.in.dt == LBI_BF16 ? backward<bf16_bits>(a, stream) : backward<float>(a, stream);
}

}  // namespace lbi
