// The selective state space scan, forward and for single tokens.
//
//   h[d,n] = exp(delta A[d,n]) h[d,n] + delta u B[n],   y = sum_n C[n] h[d,n] + D u,   times z sigmoid(z)
//
// Per row, channel and state: a product, an exponential (two issue slots: 16 of them take 1.89 ms where 16 fused products and sums take 0.94), and three
// products and sums: six slots, against four tensors of rows x channels read and written.  With 16 states that is more time on the vector
// units than in HBM: the kernel keeps them busy in all its cycles, with 40 slots a row and wave (35 instructions), of which 24 are the formula's for four
// states.  16384 x 2048 x 16: 147 us, with the states kept; 32768 x 1024 x 16: 143 us, and 98 us for the chunks' own states before it.
// Where channels and sequences alone do not fill the chip the tokens are cut into chunks: a first pass takes every chunk's
// final state from a zero one and its sum of delta (the product of its decays is exp(A * sum)), scan_carry_kernel joins them, and the
// second pass starts each chunk from its state.
#include "seq_scan.h"

namespace sn {
namespace {

constexpr int THREADS = 256;

// MODE 0: y (and, if asked for, the states of tiles and the final states); 1: the chunk's final state from zero and the sum of delta;
// 2: the states of tiles alone.
template <typename T, int NL, int WIDE, int MODE>
__global__ void __launch_bounds__(THREADS) scan_fwd_kernel(ScanArgs a)
{
    using G = ScanGeo<NL>;
    constexpr int CB = G::CB, NP = G::NP, VE = G::VE;
    constexpr bool OUT = MODE == 0, LOCAL = MODE == 1;
    // Rows staged at a time.  The loads of the next ones are on their way while these are worked on; 16 rows are too little work to cover them.
    constexpr int ROWS = 32, RP = ROWS / 16;
    __shared__ float s_delta[ROWS][CB], s_x[ROWS][CB], s_y[OUT ? ROWS : 1][OUT ? CB : 1];
    __shared__ alignas(16) float s_B[ROWS * NP];
    __shared__ alignas(16) float s_C[OUT ? ROWS * NP : 4];

    const int chunk = blockIdx.x, span = chunk / a.parts, part = chunk % a.parts;
    if (LOCAL && part == a.parts - 1) return;   // nothing comes after it
    const int group = blockIdx.y / a.blocks_per_group, inside = blockIdx.y % a.blocks_per_group * CB;
    const int c0 = group * a.per_group + inside, nch = min(CB, a.per_group - inside);
    const int r0 = span * a.span_rows + part * a.chunk_rows, r1 = min(r0 + a.chunk_rows, (span + 1) * a.span_rows);
    const ScanLane<NL> lane(a, c0, nch);
    if (OUT && chunk >= a.spans * a.parts) {
        each_empty(a.rows, chunk - a.spans * a.parts, gridDim.x - a.spans * a.parts, [&](int s) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            if (a.h0) lane.load(a.h0, s, a, v);
            lane.store(a.hT, s, a, v);
        });
        return;
    }
    const int row = threadIdx.x / 16, co = threadIdx.x % 16 * VE, nco = nch - co, nl = scan_lane() % NL;

    float bias[VE], skip[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) {
        bias[i] = a.bias && i < nco ? a.bias[c0 + co + i] : 0.f;
        skip[i] = OUT && a.D && i < nco ? a.D[c0 + co + i] : 0.f;
    }
    const char *pu = (const char *)a.u + c0 * sizeof(T), *pdt = (const char *)a.dt + c0 * sizeof(T), *pz = (const char *)a.z + c0 * sizeof(T);
    const char *pB = (const char *)a.B + group * a.N * sizeof(T), *pC = (const char *)a.C + group * a.N * sizeof(T);
    char *py = (char *)a.y + c0 * sizeof(T);
    const uint32_t is_softplus = a.softplus ? ~0u : 0u, is_gate = a.gate ? ~0u : 0u;
    float h[4] = {0.f, 0.f, 0.f, 0.f}, sum_delta = 0.f;
    bool crossed = false;
    if (!LOCAL && part > 0) lane.load_own(a.carry, chunk, a, h);

    if (r0 < r1) {
        SeqAt at = seq_find(a.rows, LOCAL ? r1 - 1 : r0);   // a chunk hands on the state of the sequence that holds its last row
        Piece next = piece_from<ROWS>(a.rows, at, LOCAL ? max(r0, at.begin) : r0, r0, r1);
        Staged<T, NL, WIDE> u[RP], dt[RP], z[RP];
        StagedBC<T, NL, ROWS, OUT, WIDE> BC;
        const auto fetch = [&]() {
            const int64_t t0 = next.t0;
            const int have = a.rows.rows - next.t0;   // rows of the tensors from there on
#pragma unroll
            for (int j = 0; j < RP; ++j) {
                const int r = min(j * 16 + row, have - 1);
                u[j].load(pu + t0 * a.ld_u, a.ld_u, r, co, nch);
                dt[j].load(pdt + t0 * a.ld_dt, a.ld_dt, r, co, nch);
                if (OUT) z[j].load(pz + t0 * a.ld_z, a.ld_z, r, co, nch);
            }
            BC.load(pB + t0 * a.ld_b, a.ld_b, pC + t0 * a.ld_c, a.ld_c, have, a.N);
        };
        float uu[RP][VE], gate[RP][VE];
        const auto stage = [&](const Piece &p) {
            const int first = p.p0 - p.t0, last = p.p1 - p.t0;
#pragma unroll
            for (int j = 0; j < RP; ++j) {
                const int r = j * 16 + row;
                const bool in = r >= first && r < last;
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    const bool here = in && i < nco;
                    const float raw = dt[j].get(i) + bias[i], delta = keep_if(here, pick(is_softplus, softplus(raw), raw));
                    uu[j][i] = keep_if(here, u[j].get(i));
                    s_delta[r][co + i] = delta;
                    s_x[r][co + i] = delta * uu[j][i];
                    if (OUT) gate[j][i] = pick(is_gate, z[j].get(i) * sigmoid(z[j].get(i)), 1.f);
                }
            }
            BC.put(s_B, s_C, first, last, a.N);
        };
        Piece now = next;
        if (now.any) {
            fetch();
            stage(now);
            next = piece_from<ROWS>(a.rows, at, now.p1, r0, r1);
            if (next.any) fetch();
        }
        __syncthreads();
        while (now.any) {
            const auto keep = [&](int t) { lane.store_own(a.states, (int64_t)span * a.tiles_per_span + (now.t0 + t - span * a.span_rows) / TS, a, h); };
            if (now.start) {
                crossed = true;
                sum_delta = 0.f;
                if (a.h0) lane.load(a.h0, now.seq, a, h);
                else h[0] = h[1] = h[2] = h[3] = 0.f;
            } else if (!LOCAL && a.states && now.p0 == now.t0) {
                keep(0);
            }

            // GR rows at a time, those of them that are not the piece's doing nothing; a row's operands are read while the one before it is worked on
            constexpr int GR = NL > 4 ? NL : 4;
            struct RowIn {
                float d, x, b[4], c[4];
            };
            const auto read = [&](int t) {
                RowIn r;
                r.d = s_delta[t][lane.c];
                r.x = s_x[t][lane.c];
                *reinterpret_cast<float4 *>(r.b) = *reinterpret_cast<const float4 *>(&s_B[t * NP + lane.n0]);
                if (OUT) *reinterpret_cast<float4 *>(r.c) = *reinterpret_cast<const float4 *>(&s_C[t * NP + lane.n0]);
                return r;
            };
            const int tb0 = (now.p0 - now.t0) / GR * GR;
            RowIn r, ahead = read(tb0);
#pragma unroll 1
            for (int tb = tb0; tb < now.p1 - now.t0; tb += GR) {
                if (!LOCAL && a.states && tb && tb % TS == 0 && now.t0 + tb > now.p0) keep(tb);
                float acc[NL];
#pragma unroll
                for (int k = 0; k < GR; ++k) {
                    r = ahead;
                    ahead = read(k + 1 < GR ? tb + k + 1 : min(tb + GR, ROWS - 1));
                    __builtin_amdgcn_sched_barrier(0x407);   // the reads stay in front: nothing but arithmetic may be moved across
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        h[i] = fmaf(exp2_fast(r.d * lane.A2[i]), h[i], r.x * r.b[i]);
                        if (OUT) sum = fmaf(h[i], r.c[i], sum);
                    }
                    acc[k % NL] = sum;
                    if (LOCAL) sum_delta += r.d;
                    if (OUT && k % NL == NL - 1) s_y[tb + k / NL * NL + nl][lane.c] = scatter_sum<NL / 2, 1>(acc);
                }
            }
            if (OUT && a.hT && now.end) lane.store(a.hT, now.seq, a, h);
            __syncthreads();
            Staged<T, NL, WIDE> y[RP];
            if (OUT)
#pragma unroll
                for (int j = 0; j < RP; ++j)
#pragma unroll
                    for (int i = 0; i < VE; ++i) y[j].set(i, fmaf(skip[i], uu[j][i], s_y[j * 16 + row][co + i]) * gate[j][i]);
            // The next rows are staged before anything is stored: whoever waits for the loads waits for what was stored since as well.
            if (next.any) stage(next);
            if (OUT)
#pragma unroll
                for (int j = 0; j < RP; ++j) {
                    const int r = j * 16 + row;
                    if (now.holds(now.t0 + r)) y[j].store(py + (int64_t)now.t0 * a.ld_y, a.ld_y, r, co, nch);
                }
            now = next;
            if (now.any) {
                next = piece_from<ROWS>(a.rows, at, now.p1, r0, r1);
                if (next.any) fetch();
            }
            __syncthreads();
        }
    }
    if (LOCAL) {
        lane.store_own(a.carry, chunk, a, h);
        if (lane.n0 == 0 && lane.there) a.sum_delta[(int64_t)chunk * a.channels + lane.channel] = sum_delta;
        if (blockIdx.y == 0 && threadIdx.x == 0) a.through[chunk] = !crossed;
    }
}

// The state that each chunk starts from, in place of the one that it ends with from zero.  Reverse: the gradient of the state that
// reaches a chunk from the one behind it.  A thread takes one value along the chunks; bound by the latency of its loads, 16 chunks' at a time.
// 1024 x 16 values through 128 chunks take 16 us (8 at a time 18; 32 need more scalar registers than there are, 56); 16 threads for
// each value, joined through LDS, take 12 there, but 51 instead of 6 where 8 sequences of 2048 x 16 values have 8 chunks each.
__global__ void __launch_bounds__(64) scan_carry_kernel(ScanArgs a, int reverse)
{
    const int64_t i = (int64_t)blockIdx.x * 64 + threadIdx.x, each = (int64_t)a.channels * a.NP;
    if (i >= each) return;
    const int channel = (int)(i / a.NP), n = (int)(i % a.NP);
    const float A2 = n < a.N ? scan_rate(a.A[(int64_t)channel * a.N + n]) : 0.f;
    const int64_t first = (int64_t)blockIdx.y * a.parts + (reverse ? a.parts - 1 : 0), dir = reverse ? -1 : 1, step = dir * each, row = dir * a.channels;
    const float *from = a.carry + first * each + i, *sums = a.sum_delta + first * a.channels + channel;
    const int *pass = a.through + first;
    float *to = a.carry + first * each + i;
    float v = 0.f;
    const auto chunks = [&](auto COUNT) {   // so many, their values on their way together
        constexpr int AT = COUNT.value;
        float local[AT], sum[AT];
        int through[AT];
#pragma unroll
        for (int k = 0; k < AT; ++k) {
            local[k] = *from;
            sum[k] = *sums;
            through[k] = *pass;
            from += step;
            sums += row;
            pass += dir;
        }
#pragma unroll
        for (int k = 0; k < AT; ++k) {
            *to = v;
            to += step;
            // The factor in two halves: between two states in range it may be beyond it (from 2^-126 to 2^127), its root is not.  A state of 0
            // stays 0, also through a root past the range (growing states before the first input).
            const float in = keep_if(through[k], v), root = keep_if(in != 0.f, exp2_fast(0.5f * (A2 * sum[k])));
            v = fmaf(root, root * in, local[k]);
        }
    };
    int k = 0;   // the last chunk hands on to nothing: it has no values
    for (; k + 16 < a.parts; k += 16) chunks(SeqInt<16>());
    for (; k + 4 < a.parts; k += 4) chunks(SeqInt<4>());
    for (; k + 1 < a.parts; ++k) chunks(SeqInt<1>());
    *to = v;
}

// One token: a thread holds four states of a channel, NL neighbouring threads a channel.  Bound by reading and writing the states: 64
// rows of 4096 x 16 9.0 us (4.0 TB/s).  WHOLE: a
// thread's four are all there, or none is.
template <typename T, int NL, bool WHOLE>
__global__ void __launch_bounds__(THREADS) scan_step_kernel(ScanArgs a, const float *state, float *state_out, const int32_t *slots, int num_slots)
{
    const int slot = step_slot(slots, blockIdx.x, num_slots);
    if (slot < 0) return;
    const int64_t t = blockIdx.x;
    const int k = blockIdx.y * THREADS + threadIdx.x, c = k / NL, n0 = k % NL * 4;
    if (c >= a.channels) return;
    const int group = c / a.per_group;
    const float *from = state + ((int64_t)slot * a.channels + c) * a.N, *A = a.A + (int64_t)c * a.N;
    float *to = state_out + ((int64_t)slot * a.channels + c) * a.N;
    const T *B = (const T *)((const char *)a.B + t * a.ld_b) + group * a.N, *C = (const T *)((const char *)a.C + t * a.ld_c) + group * a.N;
    float h[4], A2[4];   // A * log2(e) as in the kernels above: delta = 0 leaves a state as it is there and here
    Pack<T, 4> b, cc;
    if (WHOLE) {
        const int n = n0 < a.N ? n0 : 0;
        Pack<float, 4> h4, a4;
        h4.load(from + n);
        a4.load(A + n);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = h4.e[i];
            A2[i] = scan_rate(a4.e[i]);
        }
        b.load(B + n);
        cc.load(C + n);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = min(n0 + i, a.N - 1);
            h[i] = from[n];
            A2[i] = scan_rate(A[n]);
            b.e[i] = B[n];
            cc.e[i] = C[n];
        }
    }
    const float u = seq_ld<T>((const T *)((const char *)a.u + t * a.ld_u) + c), z = seq_ld<T>((const T *)((const char *)a.z + t * a.ld_z) + c);
    float raw = seq_ld<T>((const T *)((const char *)a.dt + t * a.ld_dt) + c);
    if (a.bias) raw += a.bias[c];
    const float skip = a.D ? a.D[c] : 0.f;
    const float delta = a.softplus ? softplus(raw) : raw;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[i] = fmaf(exp2_fast(delta * A2[i]), h[i], delta * u * b.get(i));
        if (n0 + i < a.N) sum = fmaf(h[i], cc.get(i), sum);
    }
    if (WHOLE) {
        Pack<float, 4> h4;
#pragma unroll
        for (int i = 0; i < 4; ++i) h4.e[i] = h[i];
        if (n0 < a.N) h4.store(to + n0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n0 + i < a.N) to[n0 + i] = h[i];
    }
#pragma unroll
    for (int m = NL / 2; m >= 1; m /= 2) sum += __shfl_xor(sum, m, 64);
    if (n0) return;
    float y = fmaf(skip, u, sum);
    if (a.gate) y *= z * sigmoid(z);
    seq_st((T *)((char *)a.y + t * a.ld_y) + c, y);
}

template <int MODE> hipError_t launch_fwd(const ScanArgs &a, const sn_scan_shape &s, const ScanPlan &p, int wide, hipStream_t st)
{
    return by_lanes_and_width(p.NL, wide, [&](auto NL, auto WIDE) {
        const dim3 grid(p.chunks + empty_groups(MODE == 0 && a.hT, a.rows), p.blocks);
        if (s.dtype == SN_BF16) scan_fwd_kernel<bf16_t, NL.value, WIDE.value, MODE><<<grid, THREADS, 0, st>>>(a);
        else scan_fwd_kernel<float, NL.value, WIDE.value, MODE><<<grid, THREADS, 0, st>>>(a);
        return hipGetLastError();
    });
}

}  // namespace

// Whether sequences of equal length share tiles and chunks, as ragged ones do, or are walked each on its own (in spans).
// On its own each has kept states for whole tiles and sums of its own, 4 KB a workgroup each; where tiles and chunks hold several, there are as many as the
// rows need.  us forward and backward, MB of kept states and workspace, 2048 channels of 16 states in bf16, each on its own and shared:
//    4096 x 4    879 +  4054, 1152       718 +  1724, 200
//    4096 x 17  1300 +  4330, 1872      1223 +  3669, 824
//     512 x 33   241 +   818,  330       274 +   757, 206
//     129 x 17    45 +   159,   58        76 +   175,  33
//    1024 x 127 1242 +  4142, 1676      1371 +  4458, 1532
// Up to a tile's length sharing is faster as soon as there are many; a few are walked side by side instead (5 x 3 rows of 832 x 16: 22 us
// forward and backward, together 45).  Beyond it, sharing saves no time but memory, and is left out where that is little: up to 8192
// workgroups own tiles and sums are at most 64 MB more, and from 128 rows on mostly less than an eighth.  A call that keeps no states
// (keeps false) has nothing to save there.
static bool shares_tiles(const sn_scan_shape &s, int blocks, bool keeps)
{
    if (s.ragged || s.rows == 0) return true;
    const int64_t len = s.rows / s.seqs, alone = (int64_t)blocks * s.seqs, tiles = (len + TS - 1) / TS;
    if (len <= TS) return alone > 1024;
    const int64_t own = tiles + (len > SUM_ROWS ? 2 : 1);   // of 4 KB: tiles, sums, what the sums have lost
    return keeps && alone > 8192 && 8 * TS * own > 9 * len;
}

ScanPlan scan_plan(const sn_scan_shape &s, int parts, bool keeps)
{
    ScanPlan p;
    p.NL = s.states <= 8 ? 2 : s.states <= 16 ? 4 : s.states <= 32 ? 8 : 16;
    p.CB = 256 / p.NL;
    p.blocks_per_group = div_up(s.channels / s.groups, p.CB);
    p.blocks = p.blocks_per_group * s.groups;
    p.spans = shares_tiles(s, p.blocks, keeps) ? 1 : s.seqs;
    p.span_rows = (int)(s.rows / p.spans);
    p.tiles_per_span = div_up(p.span_rows, TS);
    if (parts < 1) parts = 1;
    const int tiles = p.tiles_per_span ? div_up(p.tiles_per_span, parts) : 1;
    p.chunk_rows = tiles * TS;
    p.parts = p.tiles_per_span ? div_up(p.tiles_per_span, tiles) : 1;
    p.chunks = p.spans * p.parts;
    return p;
}

// Into how many chunks a span is cut when there is workspace for it.
// Whether at all: a row takes a workgroup 0.145 us (backward 0.33), alone on its compute unit or with another; cut, with the chip full of
// chunks and the pass for their own states on top, 0.46 ns (1.18 ns) go by a row and workgroup that there would be uncut, and about 14 us (10) for
// the two launches more.  us whole and cut, 16 states in bf16, 1 x 96 rows of 256 channels: 15.7, 15.3, backward 37.8, 25.9; 8 x 128 x 2048: 21.5, 31.7
// and 59.8, 68.6; 8 x 512 x 2048: 78, 79 and 189, 177; 8 x 2048 x 2048: 329, 253 and 758, 641; 16 x 2048 x 2048: 389, 473 and 1043, 1252.
// How far: a SIMD holds four waves of the forward kernels (a workgroup has one for each) and two of the backward one, and a wave alone
// leaves more than half of its issue slots empty; twice as many, so that they do not all end together; two tiles each at least.  us with 256, 512,
// 1024, 2048, 4096 workgroups: forward over 32768 x 1024 x 16 501, 320, 264, 256, 267, over 17 ragged sequences, 6000 x 2048 x 16, 209, 144, 127,
// 123, 137; forward and backward with 256, 512, 1024, 2048 in the backward pass, 8 x 2048 x 2048 x 16 1029, 943, 913, 909, 8193 x 512 x 32 335, 275, 286, 299.
int scan_parts_wanted(const sn_scan_shape &s, bool bwd, bool keeps)
{
    const ScanPlan p = scan_plan(s, 1, keeps);
    const int64_t have = (int64_t)p.blocks * p.spans, want = bwd ? 1024 : 2048;
    if ((bwd ? 280 - have : 318 - have) * p.span_rows < (bwd ? 8500 : 30000)) return 1;   // the times above, divided by the last rate
    int64_t parts = (want + have - 1) / have;
    const int64_t most = p.tiles_per_span / 2;
    if (parts > most) parts = most;
    return parts < 1 ? 1 : (int)parts;
}

size_t scan_carry_bytes(const sn_scan_shape &s, const ScanPlan &p)
{
    if (p.parts == 1) return 0;
    return align_up((size_t)p.chunks * s.channels * 4 * p.NL * 4, 256) + align_up((size_t)p.chunks * s.channels * 4, 256) + align_up((size_t)p.chunks * 4, 256);
}

ScanArgs scan_args(const sn_scan_shape &s, const ScanPlan &p, const int32_t *off, const void *u, const void *dt, const float *A, const void *B, const void *C,
                   const float *D, const void *z, const float *bias)
{
    ScanArgs a = {};
    const int64_t e = s.dtype == SN_BF16 ? 2 : 4;
    const auto bytes = [&](int64_t ld) { return s.rows > 1 ? (uint32_t)(ld * e) : 0u; };   // of a single row no stride was looked at
    a.u = u; a.dt = dt; a.A = A; a.B = B; a.C = C; a.D = D; a.z = z ? z : u; a.bias = bias; a.gate = z != nullptr;
    a.ld_u = bytes(s.ld_u); a.ld_dt = bytes(s.ld_dt); a.ld_b = bytes(s.ld_b); a.ld_c = bytes(s.ld_c); a.ld_z = bytes(z ? s.ld_z : s.ld_u); a.ld_y = bytes(s.ld_y);
    a.ld_du = bytes(s.ld_du); a.ld_ddt = bytes(s.ld_ddt); a.ld_db = bytes(s.ld_db); a.ld_dc = bytes(s.ld_dc); a.ld_dz = bytes(s.ld_dz);
    a.rows = {off, s.seqs, (int)(s.rows / s.seqs), (int)s.rows};
    a.channels = s.channels; a.N = s.states; a.NP = 4 * p.NL; a.per_group = s.channels / s.groups; a.blocks_per_group = p.blocks_per_group; a.softplus = s.softplus;
    a.span_rows = p.span_rows; a.chunk_rows = p.chunk_rows; a.parts = p.parts; a.spans = p.spans; a.tiles_per_span = p.tiles_per_span;
    return a;
}

// How rows can be staged: by the channels of a group, with four states of B and C at a time where these are whole fours.  Forward and backward over
// 3 x 517 rows in fp32, 8 states, us of the four kernels: 204 channels in two groups one by one 84, by twos 61, 208 channels by fours 57.
int scan_wide(const sn_scan_shape &s, const ScanPlan &plan)
{
    const int e = s.dtype == SN_BF16 ? 2 : 4, ve = plan.CB / 16, piece = ve * e > 16 ? 16 / e : ve, channels = s.channels / s.groups;
    return s.states % 4 ? 0 : channels % piece == 0 ? 2 : channels % 2 == 0 ? 1 : 0;
}

void scan_set_carry(ScanArgs &a, const sn_scan_shape &s, const ScanPlan &p, void *ws)
{
    char *at = (char *)ws;
    a.carry = (float *)at;
    at += align_up((size_t)p.chunks * s.channels * 4 * p.NL * 4, 256);
    a.sum_delta = (float *)at;
    at += align_up((size_t)p.chunks * s.channels * 4, 256);
    a.through = (int *)at;
}

size_t scan_states_bytes(const sn_scan_shape &s)
{
    const ScanPlan p = scan_plan(s, 1);
    return align_up((size_t)p.spans * p.tiles_per_span * s.channels * 4 * p.NL * 4, 256);
}

void scan_fwd_bytes(const sn_scan_shape &s, size_t *preferred_bytes) { *preferred_bytes = scan_carry_bytes(s, scan_plan(s, scan_parts_wanted(s, false))); }

hipError_t launch_scan_carry(const ScanArgs &a, const ScanPlan &p, bool reverse, hipStream_t st)
{
    scan_carry_kernel<<<dim3(div_up((int64_t)a.channels * a.NP, 64), p.spans), 64, 0, st>>>(a, reverse);
    return hipGetLastError();
}

template <int MODE> static hipError_t fwd_in_chunks(const ScanArgs &a, const sn_scan_shape &s, const ScanPlan &p, int wide, hipStream_t st)
{
    if (p.parts > 1) {
        hipError_t e = launch_fwd<1>(a, s, p, wide, st);
        if (e == hipSuccess) e = launch_scan_carry(a, p, false, st);
        if (e != hipSuccess) return e;
    }
    return launch_fwd<MODE>(a, s, p, wide, st);
}

hipError_t launch_scan_states(ScanArgs a, const sn_scan_shape &s, const ScanPlan &p, int wide, hipStream_t st) { return fwd_in_chunks<2>(a, s, p, wide, st); }

hipError_t launch_scan_fwd(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z, const float *bias, void *y,
                           const sn_scan_shape &s, const int32_t *off, const float *h0, float *hT, float *states, void *ws, size_t ws_bytes, hipStream_t st)
{
    const bool keeps = states != nullptr;
    ScanPlan p = scan_plan(s, scan_parts_wanted(s, false, keeps), keeps);
    while (p.parts > 1 && scan_carry_bytes(s, p) > ws_bytes) p = scan_plan(s, p.parts - 1, keeps);
    ScanArgs a = scan_args(s, p, off, u, dt, A, B, C, D, z, bias);
    a.y = y; a.h0 = h0; a.hT = hT; a.states = states;
    const int wide = scan_wide(s, p);
    if (p.parts > 1) scan_set_carry(a, s, p, ws);
    return fwd_in_chunks<0>(a, s, p, wide, st);
}

hipError_t launch_scan_step(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z, const float *bias, void *y,
                            const float *state, float *state_out, const int32_t *slots, int num_slots, const sn_scan_shape &s, hipStream_t st)
{
    const ScanPlan p = scan_plan(s, 1);
    ScanArgs a = scan_args(s, p, nullptr, u, dt, A, B, C, D, z, bias);
    a.y = y;
    const dim3 grid((int)s.rows, div_up((int64_t)s.channels * p.NL, THREADS));
    const bool whole = s.states % 4 == 0;
    return by_lanes(p.NL, [&](auto NL) {
        if (s.dtype == SN_BF16) {
            if (whole) scan_step_kernel<bf16_t, NL.value, true><<<grid, THREADS, 0, st>>>(a, state, state_out, slots, num_slots);
            else scan_step_kernel<bf16_t, NL.value, false><<<grid, THREADS, 0, st>>>(a, state, state_out, slots, num_slots);
        } else {
            if (whole) scan_step_kernel<float, NL.value, true><<<grid, THREADS, 0, st>>>(a, state, state_out, slots, num_slots);
            else scan_step_kernel<float, NL.value, false><<<grid, THREADS, 0, st>>>(a, state, state_out, slots, num_slots);
        }
        return hipGetLastError();
    });
}

}  // namespace sn
