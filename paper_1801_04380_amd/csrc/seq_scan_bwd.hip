// The gradients of the selective state space scan.
//
// With gy = dy z sigmoid(z) the gradient of the states runs backwards along the tokens,
//   g[t] = gy[t] C[t] + exp(delta[t+1] A) g[t+1],
// and everything else is made of it and of the states h:
//   du = gy D + delta sum_n g B        ddelta = u sum_n g B + sum_n A q,  q = g exp(delta A) h[t-1]        dA = sum_t delta q
//   dB = sum_d g delta u               dC = sum_d gy h
// A tile's states are computed again from the one kept before it (eight rows of states and decays in registers at a time, four states a lane),
// then the tile is walked backwards.  Three sums over a channel's states and two over a group's channels per row come on top of the
// products: scatter_sum shares an exchange among as many values as it has lanes, 8 values a row and lane for dB and dC.  The sums of a
// workgroup's channels go to the workspace and are joined by scan_join_kernel, in a fixed order.  Bound by the vector units: 118 issue slots a row
// and wave (105 instructions; exponentials and lane swaps take two slots), of which 56 are the formulas' for four states and 10 the second computation of
// the first half's states, and busy in 83 % of the cycles at two waves a SIMD (registers; four waves spill
// and are slower).  16384 x 2048 x 16: 501 us.  All 16 rows' states in registers at a time instead of eight, of which the second half's
// are computed from the state between the halves: slower, at one wave a SIMD.
// Cut into chunks like the forward pass where channels and sequences do not fill the chip: scan_bwd_local_kernel takes what a chunk hands to
// the one before it, scan_carry_kernel joins.
#include "seq_scan.h"

namespace sn {
namespace {

constexpr int THREADS = 256;

// Keeps a row's reads of LDS in front of what uses the row before it: nothing but arithmetic may be moved across.
#define ROW_AHEAD() __builtin_amdgcn_sched_barrier(0x407)

// A row's operands of a lane.
struct RowIn {
    float d, x, g, b[4], c[4];
};

// What of the gradient of the states a chunk hands on to the one before it, starting from zero, and its sum of delta.
template <typename T, int NL, int WIDE>
__global__ void __launch_bounds__(THREADS) scan_bwd_local_kernel(ScanArgs a)
{
    using G = ScanGeo<NL>;
    constexpr int CB = G::CB, NP = G::NP, VE = G::VE;
    __shared__ float s_delta[TS][CB], s_g[TS][CB];
    __shared__ alignas(16) float s_C[TS * NP];
    const int chunk = blockIdx.x, span = chunk / a.parts, part = chunk % a.parts;
    if (part == 0) return;   // nothing comes before it
    const int group = blockIdx.y / a.blocks_per_group, inside = blockIdx.y % a.blocks_per_group * CB;
    const int c0 = group * a.per_group + inside, nch = min(CB, a.per_group - inside);
    const int r0 = span * a.span_rows + part * a.chunk_rows, r1 = min(r0 + a.chunk_rows, (span + 1) * a.span_rows);
    const ScanLane<NL> lane(a, c0, nch);
    const int row = threadIdx.x / 16, co = threadIdx.x % 16 * VE, nco = nch - co;
    float bias[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) bias[i] = a.bias && i < nco ? a.bias[c0 + co + i] : 0.f;
    float g[4] = {0.f, 0.f, 0.f, 0.f}, sum_delta = 0.f;
    bool crossed = false;
    SeqAt at = seq_find(a.rows, r0);   // a chunk hands on the gradient of the sequence that holds its first row
    Piece next = piece_before<TS>(a.rows, at, min(r1, at.end), r0);
    Staged<T, NL, WIDE> dt, z, dy;
    StagedBC<T, NL, TS, false, WIDE> C;
    const char *pdt = (const char *)a.dt + c0 * sizeof(T), *pz = (const char *)a.z + c0 * sizeof(T), *pdy = (const char *)a.dy + c0 * sizeof(T);
    const char *pC = (const char *)a.C + group * a.N * sizeof(T);
    const uint32_t is_softplus = a.softplus ? ~0u : 0u, is_gate = a.gate ? ~0u : 0u;
    const auto fetch = [&]() {
        const int64_t t0 = next.t0;
        const int have = a.rows.rows - next.t0, r = min(row, have - 1);
        dt.load(pdt + t0 * a.ld_dt, a.ld_dt, r, co, nch);
        dy.load(pdy + t0 * a.ld_y, a.ld_y, r, co, nch);
        z.load(pz + t0 * a.ld_z, a.ld_z, r, co, nch);
        C.load(pC + t0 * a.ld_c, a.ld_c, nullptr, 0, have, a.N);
    };
    const auto stage = [&](const Piece &p) {
        const int first = p.p0 - p.t0, last = p.p1 - p.t0;
        const bool in = row >= first && row < last;
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const bool here = in && i < nco;
            const float raw = dt.get(i) + bias[i];
            s_delta[row][co + i] = keep_if(here, pick(is_softplus, softplus(raw), raw));
            s_g[row][co + i] = keep_if(here, dy.get(i) * pick(is_gate, z.get(i) * sigmoid(z.get(i)), 1.f));
        }
        C.put(s_C, nullptr, first, last, a.N);
    };
    Piece now = next;
    if (now.any) {
        fetch();
        stage(now);
        next = piece_before<TS>(a.rows, at, now.p0, r0);
        if (next.any) fetch();
    }
    __syncthreads();
    while (now.any) {
        if (now.end) {
            crossed = true;
            sum_delta = 0.f;
            if (a.dhT) lane.load(a.dhT, now.seq, a, g);
            else g[0] = g[1] = g[2] = g[3] = 0.f;
        }
        const auto rows = [&](int tb) {
#pragma unroll
            for (int k = 3; k >= 0; --k) {
                const float delta = s_delta[tb + k][lane.c], gy = s_g[tb + k][lane.c];
                const float4 c = *reinterpret_cast<const float4 *>(&s_C[(tb + k) * NP + lane.n0]);
                const float cc[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) g[i] = exp2_fast(delta * lane.A2[i]) * fmaf(gy, cc[i], g[i]);
                sum_delta += delta;
            }
        };
        if (now.p1 - now.p0 == TS) {
#pragma unroll
            for (int tb = TS - 4; tb >= 0; tb -= 4) rows(tb);
        } else {
            for (int tb = (now.p1 - 1 - now.t0) / 4 * 4; tb >= 0 && tb + 3 >= now.p0 - now.t0; tb -= 4) rows(tb);
        }
        __syncthreads();
        now = next;
        if (now.any) {
            stage(now);
            next = piece_before<TS>(a.rows, at, now.p0, r0);
            if (next.any) fetch();
        }
        __syncthreads();
    }
    lane.store_own(a.carry, chunk, a, g);
    if (lane.n0 == 0 && lane.there) a.sum_delta[(int64_t)chunk * a.channels + lane.channel] = sum_delta;
    if (blockIdx.y == 0 && threadIdx.x == 0) a.through[chunk] = !crossed;
}

template <typename T, int NL, int WIDE>
__global__ void __launch_bounds__(THREADS, 2) scan_bwd_kernel(ScanArgs a)
{
    using G = ScanGeo<NL>;
    constexpr int CB = G::CB, NP = G::NP, VE = G::VE, CW = G::CW;
    __shared__ float s_delta[TS][CB], s_x[TS][CB], s_g[TS][CB], s_y[TS][CB], s_qa[TS][CB], s_dD[TS][CB], s_dbias[TS][CB], s_bias[CB], s_skip[CB];
    __shared__ alignas(16) float s_B[TS * NP], s_C[TS * NP];
    __shared__ alignas(16) float s_bc[4][TS][2 * NP];

    const int chunk = blockIdx.x, span = chunk / a.parts, part = chunk % a.parts;
    const int group = blockIdx.y / a.blocks_per_group, inside = blockIdx.y % a.blocks_per_group * CB;
    const int c0 = group * a.per_group + inside, nch = min(CB, a.per_group - inside);
    const int r0 = span * a.span_rows + part * a.chunk_rows, r1 = min(r0 + a.chunk_rows, (span + 1) * a.span_rows);
    const ScanLane<NL> lane(a, c0, nch);
    const int row = threadIdx.x / 16, co = threadIdx.x % 16 * VE, nco = nch - co, nl = scan_lane() % NL, wave = threadIdx.x / 64;
    float dA[4];   // of what a thread stages, bias, D and their gradients' sums are in LDS: registers decide how many waves a SIMD has
#pragma unroll
    for (int i = 0; i < VE; ++i) {
        s_dD[row][co + i] = s_dbias[row][co + i] = 0.f;
        if (row) continue;
        s_bias[co + i] = a.bias && i < nco ? a.bias[c0 + co + i] : 0.f;
        s_skip[co + i] = a.D && i < nco ? a.D[c0 + co + i] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) dA[i] = 0.f;
    __syncthreads();
    const char *pu = (const char *)a.u + c0 * sizeof(T), *pdt = (const char *)a.dt + c0 * sizeof(T), *pz = (const char *)a.z + c0 * sizeof(T);
    const char *pdy = (const char *)a.dy + c0 * sizeof(T), *pB = (const char *)a.B + group * a.N * sizeof(T), *pC = (const char *)a.C + group * a.N * sizeof(T);
    char *pdu = (char *)a.du + c0 * sizeof(T), *pddt = (char *)a.ddt + c0 * sizeof(T), *pdz = (char *)a.dz + c0 * sizeof(T);
    float *part_bc = a.part_bc + (int64_t)blockIdx.y * a.rows.rows * (2 * NP);
    const uint32_t is_softplus = a.softplus ? ~0u : 0u, is_gate = a.gate ? ~0u : 0u;
    float g[4] = {0.f, 0.f, 0.f, 0.f};
    if (part < a.parts - 1) lane.load_own(a.carry, chunk, a, g);

    // The sums since the last time are added to what is in the workspace; those of dD and the bias's gradient over the 16 threads that stage a channel.
    bool begun = false;
    const auto add_sums = [&](bool last) {
        int at = chunk, tid = threadIdx.x;
        asm volatile("" : "+s"(at), "+v"(tid));   // addresses are formed here, not in front of the loop, through which they would take a dozen registers
        LongSum sum[4];
        float s[4] = {0.f, 0.f, 0.f, 0.f}, lost[4] = {0.f, 0.f, 0.f, 0.f};
        if (begun) {
            lane.load_own(a.part_a, at, a, s);
            lane.load_own(a.part_a + a.lost, at, a, lost);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum[i].s = s[i];
            sum[i].lost = lost[i];
            sum[i].add(dA[i]);
            s[i] = last ? sum[i].total() : sum[i].s;
            lost[i] = sum[i].lost;
            dA[i] = 0.f;
        }
        lane.store_own(a.part_a, at, a, s);
        if (!last) lane.store_own(a.part_a + a.lost, at, a, lost);
        __syncthreads();
        for (int k = tid; k < 2 * CB; k += THREADS) {
            const int c = k % CB;
            float rows = 0.f;
#pragma unroll
            for (int r = 0; r < TS; ++r) rows += k < CB ? s_dD[r][c] : s_dbias[r][c];
            if (c >= nch) continue;
            float *to = (k < CB ? a.part_d : a.part_bias) + (int64_t)at * a.channels + c0 + c;
            LongSum all;
            if (begun) {
                all.s = to[0];
                all.lost = to[a.lost];
            }
            all.add(rows);
            to[0] = last ? all.total() : all.s;
            if (!last) to[a.lost] = all.lost;
        }
        begun = true;
        if (last) return;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VE; ++i) s_dD[row][co + i] = s_dbias[row][co + i] = 0.f;
    };
    int sum_to = a.lost ? r1 - SUM_ROWS : -1;   // the row that the sums go on to

    if (r0 < r1) {
        SeqAt at = seq_find(a.rows, r1 - 1);
        Piece next = piece_before<TS>(a.rows, at, r1, r0);
        Staged<T, NL, WIDE> u, dt, z, dy;
        StagedBC<T, NL, TS, true, WIDE> BC;
        float4 kept = {};   // the state in front of the piece's tile
        const auto fetch = [&]() {
            const int64_t t0 = next.t0;
            const int have = a.rows.rows - next.t0, r = min(row, have - 1);
            u.load(pu + t0 * a.ld_u, a.ld_u, r, co, nch);
            dt.load(pdt + t0 * a.ld_dt, a.ld_dt, r, co, nch);
            dy.load(pdy + t0 * a.ld_y, a.ld_y, r, co, nch);
            z.load(pz + t0 * a.ld_z, a.ld_z, r, co, nch);
            BC.load(pB + t0 * a.ld_b, a.ld_b, pC + t0 * a.ld_c, a.ld_c, have, a.N);
            kept = lane.fetch_own(a.states, (int64_t)span * a.tiles_per_span + (next.t0 - span * a.span_rows) / TS, a);
        };
        // Of the staged piece, what its gradients take besides what is in LDS: u, d delta / d dt, d y / d z without y.  Made here, not kept as
        // loaded: a copy of what the next loads go to would have to wait for them.
        float uu[VE], slope[VE], zslope[VE];
        float first[4];   // the state in front of it
        const auto stage = [&](const Piece &p) {
            const int begin = p.p0 - p.t0, last = p.p1 - p.t0;
            const bool in = row >= begin && row < last;
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const bool here = in && i < nco;
                const float raw = dt.get(i) + s_bias[co + i], delta = keep_if(here, pick(is_softplus, softplus(raw), raw));
                const float zz = z.get(i), sz = sigmoid(zz), d = dy.get(i);
                uu[i] = keep_if(here, u.get(i));
                slope[i] = keep_if(here, pick(is_softplus, sigmoid(raw), 1.f));
                zslope[i] = d * sz * fmaf(zz, 1.f - sz, 1.f);
                s_delta[row][co + i] = delta;
                s_x[row][co + i] = delta * uu[i];
                s_g[row][co + i] = keep_if(here, pick(is_gate, d * (zz * sz), d));
            }
            BC.put(s_B, s_C, begin, last, a.N);
            lane.take(kept, a, first);
            if (p.start) {
                if (a.h0) lane.load(a.h0, p.seq, a, first);
                else first[0] = first[1] = first[2] = first[3] = 0.f;
            }
        };
        Piece now = next;
        if (now.any) {
            fetch();
            stage(now);
            next = piece_before<TS>(a.rows, at, now.p0, r0);
            if (next.any) fetch();
        }
        __syncthreads();
        int done;
        while (now.any) {   // a stretch of SUM_ROWS a turn: what adds up its sums would take registers of the loop over its pieces, if it stood in there
            do {
                if (now.end) {
                    if (a.dhT) lane.load(a.dhT, now.seq, a, g);
                    else g[0] = g[1] = g[2] = g[3] = 0.f;
                }

                constexpr int TB = CW < 8 ? 1 : CW / 8;       // rows whose 8 values share the exchanges over channels
                constexpr int GR = NL > TB ? NL : TB;         // rows that are worked on or left out together
                constexpr int HR = GR > 8 ? GR : 8;           // rows whose states are in registers at a time
                const auto read = [&](int t) {
                    RowIn r;
                    r.d = s_delta[t][lane.c];
                    r.x = s_x[t][lane.c];
                    r.g = s_g[t][lane.c];
                    *reinterpret_cast<float4 *>(r.b) = *reinterpret_cast<const float4 *>(&s_B[t * NP + lane.n0]);
                    *reinterpret_cast<float4 *>(r.c) = *reinterpret_cast<const float4 *>(&s_C[t * NP + lane.n0]);
                    return r;
                };
                const auto outside = [&](int tb, int n) { return now.t0 + tb + n <= now.p0 || now.t0 + tb >= now.p1; };
                {
                    // the state in front of the second half
                    float mid[4] = {first[0], first[1], first[2], first[3]};
                    if (HR < TS && !outside(0, HR)) {
                        RowIn r, ahead = read(0);
#pragma unroll
                        for (int t = 0; t < HR; ++t) {
                            r = ahead;
                            ahead = read(t + 1 < HR ? t + 1 : t);
                            ROW_AHEAD();
#pragma unroll
                            for (int i = 0; i < 4; ++i) mid[i] = fmaf(exp2_fast(r.d * lane.A2[i]), mid[i], r.x * r.b[i]);
                        }
                    }
#pragma unroll 1
                    for (int half = TS - HR; half >= 0; half -= HR) {
                        float hs[HR + 1][4], decay[HR][4];   // hs[k]: the state in front of the half's row k
#pragma unroll
                        for (int i = 0; i < 4; ++i) hs[0][i] = half ? mid[i] : first[i];
                        // the states, forwards; rows that are not the piece's leave them as they are
#pragma unroll
                        for (int kb = 0; kb < HR; kb += GR) {
                            float acc[NL];
                            RowIn r, ahead = read(half + kb);
#pragma unroll
                            for (int k = kb; k < kb + GR; ++k) {
                                const int t = half + k;
                                r = ahead;
                                ahead = read(k + 1 < HR ? t + 1 : t);
                                ROW_AHEAD();
                                float sum = 0.f;
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    decay[k][i] = exp2_fast(r.d * lane.A2[i]);
                                    hs[k + 1][i] = fmaf(decay[k][i], hs[k][i], r.x * r.b[i]);
                                    sum = fmaf(hs[k + 1][i], r.c[i], sum);
                                }
                                acc[t % NL] = sum;
                                if (t % NL == NL - 1) s_y[t / NL * NL + nl][lane.c] = scatter_sum<NL / 2, 1>(acc);
                            }
                        }
                        // and the gradients, backwards; what the rows' operands took in registers is read again
                        asm volatile("" ::: "memory");
#pragma unroll
                        for (int kb = HR - GR; kb >= 0; kb -= GR) {
                            if (outside(half + kb, GR)) continue;
                            float gb[NL], qa[NL], bc[8 * TB];
                            RowIn r, ahead = read(half + kb + GR - 1);
#pragma unroll
                            for (int k = kb + GR - 1; k >= kb; --k) {
                                const int t = half + k;
                                r = ahead;
                                ahead = read(k ? t - 1 : t);
                                ROW_AHEAD();
                                float sum_b = 0.f, sum_a = 0.f;
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const float gi = fmaf(r.g, r.c[i], g[i]);
                                    bc[t % TB * 8 + i] = gi * r.x;
                                    bc[t % TB * 8 + 4 + i] = r.g * hs[k + 1][i];
                                    sum_b = fmaf(gi, r.b[i], sum_b);
                                    g[i] = decay[k][i] * gi;
                                    const float q = g[i] * hs[k][i];
                                    sum_a = fmaf(q, lane.A2[i], sum_a);
                                    dA[i] = fmaf(q, r.d, dA[i]);
                                }
                                gb[t % NL] = sum_b;
                                qa[t % NL] = sum_a;
                                if (t % NL == 0) {   // rows t .. t + NL - 1 are done
                                    s_x[t + nl][lane.c] = scatter_sum<NL / 2, 1>(gb);   // over what the rows were staged with
                                    s_qa[t + nl][lane.c] = scatter_sum<NL / 2, 1>(qa);
                                }
                                if (t % TB == 0) {
                                    const int k8 = scan_lane() / NL;   // which of the rows' values this lane gets
                                    if constexpr (CW >= 8) {
                                        s_bc[wave][t + k8 / 8][(k8 / 4 & 1) * NP + lane.n0 + k8 % 4] = scatter_sum<32, NL>(bc);
                                    } else {
                                        float lo[4] = {bc[0], bc[1], bc[2], bc[3]}, hi[4] = {bc[4], bc[5], bc[6], bc[7]};
                                        s_bc[wave][t][lane.n0 + k8] = scatter_sum<32, NL>(lo);
                                        s_bc[wave][t][NP + lane.n0 + k8] = scatter_sum<32, NL>(hi);
                                    }
                                }
                            }
                        }
                    }
                }
                if (a.dh0 && now.start) lane.store(a.dh0, now.seq, a, g);
                __syncthreads();
                const bool in = now.holds(now.t0 + row);
                Staged<T, NL, WIDE> du, ddt, dz;
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    const float vb = s_x[row][co + i], va = s_qa[row][co + i] * 0.69314718055994530942f /* A is A2 * ln 2 */, gy = s_g[row][co + i];
                    const float dd = fmaf(uu[i], vb, va) * slope[i];
                    du.set(i, fmaf(gy, s_skip[co + i], s_delta[row][co + i] * vb));
                    ddt.set(i, dd);
                    dz.set(i, zslope[i] * fmaf(s_skip[co + i], uu[i], s_y[row][co + i]));
                    const bool here = in && i < nco;
                    s_dbias[row][co + i] += keep_if(here, dd);
                    s_dD[row][co + i] = fmaf(gy, uu[i], s_dD[row][co + i]);   // both are zero elsewhere
                }
                constexpr int PER = (TS * 2 * NP / 4 + THREADS - 1) / THREADS;
                float4 bc[PER];
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int k = i * THREADS + threadIdx.x, r = k * 4 / (2 * NP) % TS, n = k * 4 % (2 * NP);
                    const auto at = [&](int w) { return *reinterpret_cast<const float4 *>(&s_bc[w][r][n]); };
                    const float4 p = at(0), q = at(1), v = at(2), w = at(3);
                    bc[i] = make_float4(p.x + q.x + v.x + w.x, p.y + q.y + v.y + w.y, p.z + q.z + v.z + w.z, p.w + q.w + v.w + w.w);
                }
                // The next rows are staged before anything is stored: whoever waits for the loads waits for what was stored since as well.
                if (next.any) stage(next);
                if (in) {
                    du.store(pdu + (int64_t)now.t0 * a.ld_du, a.ld_du, row, co, nch);
                    ddt.store(pddt + (int64_t)now.t0 * a.ld_ddt, a.ld_ddt, row, co, nch);
                    if (a.gate) dz.store(pdz + (int64_t)now.t0 * a.ld_dz, a.ld_dz, row, co, nch);
                }
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const uint32_t k = i * THREADS + threadIdx.x, r = k * 4 / (2 * NP);
                    if (r < TS && now.holds(now.t0 + r)) *reinterpret_cast<float4 *>(part_bc + (int64_t)now.t0 * (2 * NP) + k * 4) = bc[i];
                }
                done = now.p0;
                now = next;
                if (now.any) {
                    next = piece_before<TS>(a.rows, at, now.p0, r0);
                    if (next.any) fetch();
                }
                __syncthreads();
            } while (now.any && done > sum_to);
            if (!now.any) break;
            sum_to = done - SUM_ROWS;
            add_sums(false);
        }
    }
    add_sums(true);
}

// dB and dC from the sums of the channel blocks: one thread per row, group, tensor and state, k counts them.
template <typename T> __device__ inline void join_bc(const ScanArgs &a, int groups, int64_t k)
{
    const int n = (int)(k % a.NP), which = (int)(k / a.NP % 2), group = (int)(k / (2 * a.NP) % groups);
    const int64_t row = k / (2 * a.NP) / groups;
    if (row >= a.rows.rows || n >= a.N) return;
    if (a.rows.off && !seq_find(a.rows, (int)row).holds((int)row, a.rows)) return;
    float sum = 0.f;
    for (int b = 0; b < a.blocks_per_group; ++b)
        sum += a.part_bc[(((int64_t)group * a.blocks_per_group + b) * a.rows.rows + row) * (2 * a.NP) + which * a.NP + n];
    char *to = which ? (char *)a.dC + row * a.ld_dc : (char *)a.dB + row * a.ld_db;
    seq_st((T *)to + group * a.N + n, sum);
}

// The gradients of empty sequences' states: of those that a group looks at, SLICE elements.
constexpr int SLICE = 16 * THREADS;
__device__ inline void pass_empty(const ScanArgs &a, int group, int count, int slice)
{
    const int64_t each = (int64_t)a.channels * a.N;
    each_empty(a.rows, group, count, [&](int s) {
#pragma unroll 4
        for (int k = threadIdx.x; k < SLICE; k += THREADS) {
            const int64_t i = (int64_t)slice * SLICE + k;
            if (i < each) a.dh0[s * each + i] = a.dhT ? a.dhT[s * each + i] : 0.f;
        }
    });
}

// What is left to join, in one launch: the first `sums` workgroups take dA, dD and the bias's gradient from the sums of the chunks, 16 threads
// along the chunks of each value, joined in a fixed order; the next `bcs` dB and dC; the others, `empties` for each slice of a state, dh0 of empty sequences.
template <typename T>
__global__ void __launch_bounds__(THREADS) scan_join_kernel(ScanArgs a, int groups, int chunks, unsigned sums, int64_t bcs, int empties, float *__restrict__ dA,
                                                            float *__restrict__ dD, float *__restrict__ dbias)
{
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (block >= sums + bcs) {
        const int64_t k = block - sums - bcs;
        if (empties) pass_empty(a, (int)(k % empties), empties, (int)(k / empties));
        return;
    }
    if (block >= sums) {
        join_bc<T>(a, groups, (block - sums) * THREADS + threadIdx.x);
        return;
    }
    __shared__ float lds[16][16];
    const int lane = threadIdx.x / 16;
    const int64_t i = block * 16 + threadIdx.x % 16, each = (int64_t)a.channels * a.N;
    const float *from = a.part_a;
    float *to = nullptr;
    int64_t at = 0, stride = a.channels;
    if (i < each) { from = a.part_a + i / a.N * (a.NP - a.N); to = dA; at = i; stride = (int64_t)a.channels * a.NP; }
    else if (i < each + a.channels) { from = a.part_d; to = dD; at = i - each; }
    else if (i < each + 2 * (int64_t)a.channels) { from = a.part_bias; to = dbias; at = i - each - a.channels; }
    LongSum sum, all;
    if (to)
#pragma unroll 8
        for (int c = lane; c < chunks; c += 16) sum.add(from[c * stride + at]);
    lds[lane][threadIdx.x % 16] = sum.total();
    __syncthreads();
    if (lane || !to) return;
#pragma unroll
    for (int c = 0; c < 16; ++c) all.add(lds[c][threadIdx.x]);
    to[at] = all.total();
}

template <typename T, int NL, int WIDE> hipError_t bwd_in_chunks(const ScanArgs &a, const ScanPlan &p, hipStream_t st)
{
    const dim3 grid(p.chunks, p.blocks);
    if (p.parts > 1) {
        scan_bwd_local_kernel<T, NL, WIDE><<<grid, THREADS, 0, st>>>(a);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess) e = launch_scan_carry(a, p, true, st);
        if (e != hipSuccess) return e;
    }
    scan_bwd_kernel<T, NL, WIDE><<<grid, THREADS, 0, st>>>(a);
    return hipGetLastError();
}

struct BwdBytes {
    size_t carry, a, d, lost, bc;
    size_t all() const { return carry + a + 2 * d + lost + bc; }
};

BwdBytes bytes_of(const sn_scan_shape &s, const ScanPlan &p)
{
    BwdBytes b;
    b.carry = scan_carry_bytes(s, p);
    b.a = align_up((size_t)p.chunks * s.channels * 4 * p.NL * 4, 256);
    b.d = align_up((size_t)p.chunks * s.channels * 4, 256);
    b.lost = p.chunk_rows > SUM_ROWS ? b.a + 2 * b.d : 0;
    b.bc = align_up((size_t)p.blocks * s.rows * 8 * p.NL * 4, 256);
    return b;
}

}  // namespace

void scan_bwd_bytes(const sn_scan_shape &s, size_t *min_bytes, size_t *preferred_bytes)
{
    *min_bytes = bytes_of(s, scan_plan(s, 1)).all();
    *preferred_bytes = bytes_of(s, scan_plan(s, scan_parts_wanted(s, true))).all();
}

hipError_t launch_scan_bwd(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z, const float *bias,
                           const ScanGrads &g, const sn_scan_shape &s, const int32_t *off, const float *h0, const float *states, void *ws, size_t ws_bytes, hipStream_t st)
{
    const size_t replay = states ? 0 : scan_states_bytes(s);
    ScanPlan p = scan_plan(s, scan_parts_wanted(s, true));
    while (p.parts > 1 && replay + bytes_of(s, p).all() > ws_bytes) p = scan_plan(s, p.parts - 1);
    const BwdBytes b = bytes_of(s, p);
    ScanArgs a = scan_args(s, p, off, u, dt, A, B, C, D, z, bias);
    a.h0 = h0;
    a.dy = g.dy; a.du = g.du; a.ddt = g.ddt; a.dB = g.dB; a.dC = g.dC; a.dz = g.dz; a.dhT = g.dhT; a.dh0 = g.dh0;
    const int wide = scan_wide(s, p);
    char *at = (char *)ws;
    a.states = states ? const_cast<float *>(states) : (float *)at;
    at += replay;
    if (p.parts > 1) scan_set_carry(a, s, p, at);
    at += b.carry;
    a.part_a = (float *)at; at += b.a;
    a.part_d = (float *)at; at += b.d;
    a.part_bias = (float *)at; at += b.d;
    a.lost = b.lost / 4; at += b.lost;
    a.part_bc = (float *)at;
    hipError_t e = hipSuccess;
    if (!states && s.rows) e = launch_scan_states(a, s, p, wide, st);
    if (e != hipSuccess) return e;
    const bool bf16 = s.dtype == SN_BF16;
    e = by_lanes_and_width(p.NL, wide, [&](auto NL, auto WIDE) {
        return bf16 ? bwd_in_chunks<bf16_t, NL.value, WIDE.value>(a, p, st) : bwd_in_chunks<float, NL.value, WIDE.value>(a, p, st);
    });
    if (e != hipSuccess) return e;
    const int64_t sums = ((int64_t)s.channels * (s.states + 2) + 15) / 16, bcs = (s.rows * s.groups * 8 * p.NL + THREADS - 1) / THREADS;
    const int empties = empty_groups(g.dh0, a.rows);
    const int64_t all = sums + bcs + (int64_t)empties * div_up((int64_t)s.channels * s.states, SLICE);
    const int64_t most = 1 << 20;   // in x: a dimension of a grid has to stay below 2^32 threads
    const dim3 blocks((unsigned)(all < most ? all : most), (unsigned)((all + most - 1) / most));
    if (bf16) scan_join_kernel<bf16_t><<<blocks, THREADS, 0, st>>>(a, s.groups, p.chunks, (unsigned)sums, bcs, empties, g.dA, g.dD, g.ddt_bias);
    else scan_join_kernel<float><<<blocks, THREADS, 0, st>>>(a, s.groups, p.chunks, (unsigned)sums, bcs, empties, g.dA, g.dD, g.ddt_bias);
    return hipGetLastError();
}

}  // namespace sn
