// What the scan's kernels share.
//
// A workgroup of four waves works on CB channels of one group and walks along the tokens in tiles of TS rows.  A lane holds four states of
// one channel: NL lanes (2, 4, 8 or 16 for up to 8, 16, 32, 64 states) hold a channel's, the wave 64 / NL channels.  Sums over a channel's
// states then are four products in a lane and log2(NL) exchanges, shared by NL rows (scatter_high); sums over channels, which only
// the gradients of B and C need, are exchanges among the 64 / NL lanes of a wave, shared by as many values (scatter_low).
// Rows are staged through LDS by all threads: delta, delta * u and the rest of what is per row and channel is computed once, not in every
// lane of a channel.
#pragma once
#include "seq.h"

namespace sn {

constexpr int TS = 16;   // rows of a tile, and between two kept states

template <int NL> struct ScanGeo {
    static constexpr int CW = 64 / NL, CB = 4 * CW, NP = 4 * NL;
    static constexpr int VE = CB / 16;                                  // a thread stages VE neighbouring channels of row tid / 16
    template <typename T> static constexpr int piece() { return VE * (int)sizeof(T) > 16 ? 16 / (int)sizeof(T) : VE; }   // in one access
};

struct ScanArgs {
    const void *u, *dt, *B, *C, *z, *dy;
    const float *A, *D, *bias;
    void *y, *du, *ddt, *dB, *dC, *dz;
    int64_t ld_u, ld_dt, ld_b, ld_c, ld_z, ld_y, ld_du, ld_ddt, ld_db, ld_dc, ld_dz;
    const float *h0, *dhT;
    float *hT, *dh0, *states;
    SeqRows rows;
    int channels, N, per_group, blocks_per_group, softplus;
    int span_rows, chunk_rows, parts, spans, tiles_per_span;  // a span (a sequence, or all rows) in `parts` chunks
    float *carry, *sum_delta;                                 // [chunk][channels][N], [chunk][channels]
    int *through;                                             // [chunk]: no sequence ends and begins in it
    float *part_a, *part_d, *part_bias, *part_bc;             // sums of chunks; of channel blocks [block][row][2][NP]
    int whole_u, whole_dt, whole_z, whole_y, whole_du, whole_ddt, whole_dz;
};

// Whether a tile's rows are in a sequence, its first or its last, a bit each; and the sequence, lane i's for row i.
struct TileAt {
    unsigned valid, start, end;
    int seq;
    __device__ int of(int i) const { return __shfl(seq, i, 64); }
};

// The tile of rows t0 .. r1 - 1 at most.  `at`: the place of some row near it, whose sequence most tiles lie in.
__device__ inline TileAt tile_at(const SeqRows &r, SeqAt &at, int t0, int r1, bool keep_last)
{
    const int last = min(t0 + TS, r1), lane = threadIdx.x & 63;
    TileAt m;
    if (at.s >= 0 && at.s < r.seqs && at.begin <= t0 && last <= at.end) {
        m.valid = (1u << (last - t0)) - 1u;
        m.start = t0 == at.begin;
        m.end = last == at.end ? 1u << (last - t0 - 1) : 0u;
        m.seq = at.s;
        return m;
    }
    const int row = t0 + lane;
    SeqAt mine = at;
    bool in = false;
    if (row < last) {
        mine = seq_find(r, row);
        in = mine.holds(row, r);
    }
    m.valid = (unsigned)__ballot(in);
    m.start = (unsigned)__ballot(in && row == mine.begin);
    m.end = (unsigned)__ballot(in && row == mine.end - 1);
    m.seq = mine.s;
    const int from = keep_last ? last - t0 - 1 : 0;
    at.s = __builtin_amdgcn_readlane(mine.s, from);
    at.begin = __builtin_amdgcn_readlane(mine.begin, from);
    at.end = __builtin_amdgcn_readlane(mine.end, from);
    return m;
}

// a[lane < 32], b[lane >= 32] with their partners' added: one swap and one addition for two values
__device__ inline float fold32(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// the same for lanes 16 apart
__device__ inline float fold16(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int M> __device__ inline float fold_low(float a, float b)
{
    const bool up = (threadIdx.x & M) != 0;
    const float keep = up ? b : a, give = up ? a : b;
    return keep + __shfl_xor(give, M, 64);
}
template <int M> __device__ inline float fold(float a, float b)
{
    if constexpr (M == 32) return fold32(a, b);
    else if constexpr (M == 16) return fold16(a, b);
    else return fold_low<M>(a, b);
}

// v[i] summed over the lanes that differ in the bits from TOP down to LOW; the lane whose bits there read i gets sum i.
template <int TOP, int LOW, int COUNT> __device__ inline float scatter_sum(float (&v)[COUNT])
{
    static_assert(COUNT == 2 * TOP / LOW, "a value for each lane");
#pragma unroll
    for (int i = 0; i < COUNT / 2; ++i) v[i] = fold<TOP>(v[i], v[i + COUNT / 2]);
    if constexpr (TOP > LOW) {
        float w[COUNT / 2];
#pragma unroll
        for (int i = 0; i < COUNT / 2; ++i) w[i] = v[i];
        return scatter_sum<TOP / 2, LOW, COUNT / 2>(w);
    } else {
        return v[0];
    }
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }   // v_exp_f32; results below 2^-126 are 0

__device__ inline float softplus(float x) { return x > 20.f ? x : log1pf(expf(x)); }   // log(1 + e^-20) is below half a step of 20

// The lane's channel of a group's block, its states, and what is fixed of them.
template <int NL> struct ScanLane {
    int c, n0, channel;   // channel within the workgroup's, first state, channel of the tensors
    bool there;
    float A2[4];          // A * log2(e)
    __device__ ScanLane(const ScanArgs &a, int c0, int nch)
    {
        constexpr int CW = ScanGeo<NL>::CW;
        const int lane = threadIdx.x & 63;
        c = (threadIdx.x / 64) * CW + lane % CW;
        n0 = lane / CW * 4;
        there = c < nch;
        channel = c0 + c;
#pragma unroll
        for (int i = 0; i < 4; ++i) A2[i] = there && n0 + i < a.N ? a.A[(int64_t)channel * a.N + n0 + i] * 1.44269504088896340736f : 0.f;
    }
    // four states of array p, [..][channels][N], at index k of its first dimension
    __device__ void load(const float *p, int64_t k, const ScanArgs &a, float (&v)[4]) const
    {
        const float *q = p + (k * a.channels + channel) * a.N + n0;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = there && n0 + i < a.N ? q[i] : 0.f;
    }
    __device__ void store(float *p, int64_t k, const ScanArgs &a, const float (&v)[4]) const
    {
        float *q = p + (k * a.channels + channel) * a.N + n0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (there && n0 + i < a.N) q[i] = v[i];
    }
};

// VE neighbouring channels of a row, as they lie in memory.
template <typename T, int NL> struct Staged {
    static constexpr int P = ScanGeo<NL>::template piece<T>(), PN = ScanGeo<NL>::VE / P;
    Pack<T, P> p[PN];
    __device__ void load(const void *base, int64_t at, int n, bool whole)
    {
#pragma unroll
        for (int i = 0; i < PN; ++i) p[i].load((const T *)base + at + i * P, n - i * P, whole);
    }
    __device__ void store(void *base, int64_t at, int n, bool whole) const
    {
#pragma unroll
        for (int i = 0; i < PN; ++i) p[i].store((T *)base + at + i * P, n - i * P, whole);
    }
    __device__ void zero()
    {
#pragma unroll
        for (int i = 0; i < PN; ++i) p[i].zero();
    }
    __device__ float get(int i) const { return p[i / P].get(i % P); }
    __device__ void set(int i, float v) { p[i / P].set(i % P, v); }
};

// A row's B or C of one group: NP values, a thread's share of a tile.
template <typename T, int NL> struct StagedBC {
    static constexpr int COUNT = TS * ScanGeo<NL>::NP, PER = (COUNT + 255) / 256;
    T v[PER];
    __device__ void load(const void *base, int64_t ld, int t0, int64_t column, int N, unsigned valid)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int k = i * 256 + threadIdx.x, row = k / ScanGeo<NL>::NP, n = k % ScanGeo<NL>::NP;
            v[i] = k < COUNT && n < N && (valid >> row & 1) ? ((const T *)base)[(int64_t)(t0 + row) * ld + column + n] : (T)0;
        }
    }
    __device__ void put(float *lds) const
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int k = i * 256 + threadIdx.x;
            if (k < COUNT) lds[k] = seq_ld<T>(&v[i]);
        }
    }
};

// ---- host side ----
// How a call is laid out: the lanes of a channel, the channel blocks, and the chunks that the spans are cut into.
struct ScanPlan {
    int NL, CB, blocks_per_group, blocks;
    int spans, span_rows, chunk_rows, parts, chunks, tiles_per_span;
};
ScanPlan scan_plan(const sn_scan_shape &s, int parts);
int scan_parts_wanted(const sn_scan_shape &s, bool bwd);
size_t scan_carry_bytes(const sn_scan_shape &s, const ScanPlan &p);
ScanArgs scan_args(const sn_scan_shape &s, const ScanPlan &p, const int32_t *off);
int scan_whole_rows(const void *p, int64_t ld, const sn_scan_shape &s, const ScanPlan &plan);
void scan_set_carry(ScanArgs &a, const sn_scan_shape &s, const ScanPlan &p, void *ws);
hipError_t launch_scan_states(ScanArgs a, const sn_scan_shape &s, const ScanPlan &p, hipStream_t st);   // a.states from the inputs
hipError_t launch_scan_carry(const ScanArgs &a, const ScanPlan &p, bool reverse, hipStream_t st);

template <int V> struct ScanInt { static constexpr int value = V; };
template <typename F> hipError_t by_lanes(int NL, F f)
{
    return NL == 2 ? f(ScanInt<2>()) : NL == 4 ? f(ScanInt<4>()) : NL == 8 ? f(ScanInt<8>()) : f(ScanInt<16>());
}

}  // namespace sn
