// What the scan's kernels share.
//
// A workgroup of four waves works on CB channels of one group and walks along the tokens in tiles of TS rows.  A lane holds four states of
// one channel: NL neighbouring lanes (2, 4, 8 or 16 for up to 8, 16, 32, 64 states) hold a channel's, the wave 64 / NL channels.  Sums
// over a channel's states then are four products in a lane and log2(NL) exchanges, shared by NL rows; sums over channels, which only the
// gradients of B and C need, are exchanges among the lanes of like states, shared by 64 / NL values (scatter_sum).  The latter are the
// more, so they have the bits of the lane number that exchange by lane swaps: two instructions a pair and not three, though as many issue slots, as
// a swap takes two of them.
// Rows are staged through LDS by all threads: delta, delta * u and the rest of what is per row and channel is computed once, not in every
// lane of a channel.
#pragma once
#include "seq.h"

namespace sn {

constexpr int TS = 16;   // rows between two kept states; of a tile in the backward pass
// Rows (and up to a tile more) after which the gradients' sums over rows start from zero again, and what they were is added to what is in the workspace without loss.  A
// running sum of n terms is off by up to n * 2^-24 of them (over 2^20 equal rows dA was off by 0.6 %); like this by 2^-16 at most, and by about 2^-21 where
// the roundings are as often up as down.
constexpr int SUM_ROWS = 256;

template <int NL> struct ScanGeo {
    static constexpr int CW = 64 / NL, CB = 4 * CW, NP = 4 * NL;
    static constexpr int VE = CB / 16;                                  // a thread stages VE neighbouring channels of row tid / 16
    template <typename T> static constexpr int piece() { return VE * (int)sizeof(T) > 16 ? 16 / (int)sizeof(T) : VE; }   // in one access
};

struct ScanArgs {
    const void *u, *dt, *B, *C, *z, *dy;
    const float *A, *D, *bias;
    void *y, *du, *ddt, *dB, *dC, *dz;
    uint32_t ld_u, ld_dt, ld_b, ld_c, ld_z, ld_y, ld_du, ld_ddt, ld_db, ld_dc, ld_dz;   // row strides in bytes, 2^26 at most
    const float *h0, *dhT;
    float *hT, *dh0, *states;
    SeqRows rows;
    int channels, N, per_group, blocks_per_group, softplus;
    int span_rows, chunk_rows, parts, spans, tiles_per_span;  // a span (a long sequence, or all rows) in `parts` chunks
    float *carry, *sum_delta;                                 // [chunk][channels][NP], [chunk][channels]
    int *through;                                             // [chunk]: no sequence ends and begins in it
    int NP;                                                   // the states of the library's own arrays: padded to four for each lane
    float *part_a, *part_d, *part_bias, *part_bc;             // sums of chunks; of channel blocks [block][row][2][NP]
    int64_t lost;   // what the sums of chunks have lost so far is so many elements behind each of them; 0: chunks of SUM_ROWS at most, whose sums are added once
    int gate;   // z is there; if not, z is u: loaded and left out
};

// Lanes are numbered so that every bit of the number can be flipped by one cross-lane operand: bits 5 and 4 by the lane swaps, 3 by row_ror:8,
// 1 and 0 by quad_perm.  For bit 2 there is only the mirror among eight lanes, which flips bits 1 and 0 of the hardware's
// number as well; these two are therefore counted inverted where bit 2 is set.
__device__ inline int scan_lane()
{
    const int lane = threadIdx.x & 63;
    return lane & 4 ? lane ^ 3 : lane;
}

// Of two values the one that belongs to this lane's bit M (a: clear, b: set), with the other lane's added.
template <int M> __device__ inline float fold(float a, float b)
{
    if constexpr (M == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else if constexpr (M == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else {
        constexpr int how = M == 8 ? 0x128 /* row_ror:8 */ : M == 4 ? 0x141 /* row_half_mirror */ : M == 2 ? 0x4e /* quad_perm:[2,3,0,1] */ : 0xb1 /* quad_perm:[1,0,3,2] */;
        const bool up = (scan_lane() & M) != 0;
        const float keep = up ? b : a, give = up ? a : b;
        return keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(give), how, 0xf, 0xf, true));
    }
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

// A * log2(e), held within the range: 0 * A has to stay 0 in rows that are not the piece's, also for A = -inf, where all others decay to 0.
__device__ inline float scan_rate(float A)
{
    const float A2 = A * 1.44269504088896340736f;
    return A2 == -INFINITY ? -3.402823466e38f : A2;
}

// The lane's channel of a group's block, its states, and what is fixed of them.
template <int NL> struct ScanLane {
    int c, n0, channel;   // channel within the workgroup's, first state, channel of the tensors
    bool there;
    float A2[4];          // A * log2(e)
    __device__ ScanLane(const ScanArgs &a, int c0, int nch)
    {
        const int lane = scan_lane();
        c = (threadIdx.x / 64) * ScanGeo<NL>::CW + lane / NL;
        n0 = lane % NL * 4;
        there = c < nch;
        channel = c0 + c;
#pragma unroll
        for (int i = 0; i < 4; ++i) A2[i] = there && n0 + i < a.N ? scan_rate(a.A[(int64_t)channel * a.N + n0 + i]) : 0.f;
    }
    // Four states of one of the library's own arrays, [..][channels][NP]: padded, so that they are one access.  In two steps: a load without a
    // condition, and the choice of what is there.
    __device__ float4 fetch_own(const float *p, int64_t k, const ScanArgs &a) const
    {
        return *reinterpret_cast<const float4 *>(p + (k * a.channels + (there ? channel : channel - c)) * ScanGeo<NL>::NP + n0);
    }
    __device__ void take(const float4 &q, const ScanArgs &a, float (&v)[4]) const
    {
        v[0] = there && n0 < a.N ? q.x : 0.f;
        v[1] = there && n0 + 1 < a.N ? q.y : 0.f;
        v[2] = there && n0 + 2 < a.N ? q.z : 0.f;
        v[3] = there && n0 + 3 < a.N ? q.w : 0.f;
    }
    __device__ void load_own(const float *p, int64_t k, const ScanArgs &a, float (&v)[4]) const { take(fetch_own(p, k, a), a, v); }
    __device__ void store_own(float *p, int64_t k, const ScanArgs &a, const float (&v)[4]) const
    {
        if (there) *reinterpret_cast<float4 *>(p + (k * a.channels + channel) * ScanGeo<NL>::NP + n0) = make_float4(v[0], v[1], v[2], v[3]);
    }
    // Four states of array p, [..][channels][N], at index k of its first dimension.  The choice of what is there waits for them, so that nothing
    // has to where the ways from a call under a condition meet.
    __device__ void load(const float *p, int64_t k, const ScanArgs &a, float (&v)[4]) const
    {
        const float *q = p + (k * a.channels + (there ? channel : channel - c)) * a.N;
        take(make_float4(q[min(n0, a.N - 1)], q[min(n0 + 1, a.N - 1)], q[min(n0 + 2, a.N - 1)], q[min(n0 + 3, a.N - 1)]), a, v);
    }
    __device__ void store(float *p, int64_t k, const ScanArgs &a, const float (&v)[4]) const
    {
        float *q = p + (k * a.channels + channel) * a.N + n0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (there && n0 + i < a.N) q[i] = v[i];
    }
};

// Choices as one instruction and no branch, which would cut the code around it into pieces that nothing is moved across: v or zero; a where the
// mask is all ones, b where it is zero.
__device__ inline float keep_if(bool here, float v) { return __uint_as_float(__float_as_uint(v) & (here ? ~0u : 0u)); }
__device__ inline float pick(uint32_t mask, float a, float b) { return __uint_as_float((__float_as_uint(a) & mask) | (__float_as_uint(b) & ~mask)); }

// VE neighbouring channels of a row, as they lie in memory: of the nch channels that a row of the tile at `tile` begins with (the place of its
// first row, the same for all lanes: the lane's part of an address is 32 bits) those from co on.  WIDE 2, 1, 0: in pieces of up to
// 16 bytes, by twos (a piece's channels are all there or none is), one by one.
template <typename T, int NL, int WIDE> struct Staged {
    static constexpr int VE = ScanGeo<NL>::VE, P = WIDE == 2 ? ScanGeo<NL>::template piece<T>() : WIDE && VE > 1 ? 2 : 1, PN = VE / P;
    Pack<T, P> p[PN];
    __device__ void load(const char *tile, uint32_t ld, int row, int co, int nch)
    {
#pragma unroll
        for (int i = 0; i < PN; ++i) {
            const int c = WIDE ? (co + i * P < nch ? co + i * P : 0) : min(co + i, nch - 1);
            p[i].load(reinterpret_cast<const T *>(tile + (uint32_t)(row * ld + c * (uint32_t)sizeof(T))));
        }
    }
    __device__ void store(char *tile, uint32_t ld, int row, int co, int nch) const
    {
#pragma unroll
        for (int i = 0; i < PN; ++i)
            if (co + i * P < nch) p[i].store(reinterpret_cast<T *>(tile + (uint32_t)(row * ld + (co + i * P) * (uint32_t)sizeof(T))));
    }
    __device__ float get(int i) const { return p[i / P].get(i % P); }
    __device__ void set(int i, float v) { p[i / P].set(i % P, v); }
};

// The rows of B and C of one group, NP values each, a thread's share of a tile of which the first `have` rows are in the tensors.  WIDE: four
// neighbouring states at a time, so that a wave or two load what all four would one by one.  first .. last - 1: the rows of the piece, the
// others are staged as zeros.
template <typename T, int NL, int ROWS, bool BOTH, int WIDE> struct StagedBC {
    static constexpr int NP = ScanGeo<NL>::NP, V = WIDE ? 4 : 1, EACH = ROWS * NP / V, COUNT = (BOTH ? 2 : 1) * EACH, PER = (COUNT + 255) / 256;
    Pack<T, V> v[PER];
    // B, C: the tile's first rows; the first alone unless BOTH
    __device__ void load(const char *B, uint32_t ld_b, const char *C, uint32_t ld_c, int have, int N)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int k = i * 256 + threadIdx.x, r = min(k % EACH * V / NP, have - 1), n = k * V % NP;
            const uint32_t at = (uint32_t)(WIDE ? (n < N ? n : 0) : min(n, N - 1)) * (uint32_t)sizeof(T);
            v[i].load(reinterpret_cast<const T *>(BOTH && k / EACH % 2 ? C + (uint32_t)(r * ld_c + at) : B + (uint32_t)(r * ld_b + at)));
        }
    }
    __device__ void put(float *s_B, float *s_C, int first, int last, int N) const
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int k = i * 256 + threadIdx.x, w = k % EACH, r = w * V / NP, n = k * V % NP;
            if (k >= COUNT) continue;
            float *to = (BOTH && k >= EACH ? s_C : s_B) + w * V;
            const bool here = r >= first && r < last;
            if (WIDE) {
                const bool in = here && n < N;
                *reinterpret_cast<float4 *>(to) = make_float4(keep_if(in, v[i].get(0)), keep_if(in, v[i].get(V > 1 ? 1 : 0)), keep_if(in, v[i].get(V > 1 ? 2 : 0)), keep_if(in, v[i].get(V > 1 ? 3 : 0)));
            } else {
                to[0] = keep_if(here && n < N, v[i].get(0));
            }
        }
    }
};

// ---- host side ----
// How a call is laid out: the lanes of a channel, the channel blocks, and the chunks that the spans are cut into.
struct ScanPlan {
    int NL, CB, blocks_per_group, blocks;
    int spans, span_rows, chunk_rows, parts, chunks, tiles_per_span;
};
ScanPlan scan_plan(const sn_scan_shape &s, int parts, bool keeps = true);   // keeps: states of tiles are kept, or made for the gradient
int scan_parts_wanted(const sn_scan_shape &s, bool bwd, bool keeps = true);
size_t scan_carry_bytes(const sn_scan_shape &s, const ScanPlan &p);
ScanArgs scan_args(const sn_scan_shape &s, const ScanPlan &p, const int32_t *off, const void *u, const void *dt, const float *A, const void *B, const void *C,
                   const float *D, const void *z, const float *bias);
int scan_wide(const sn_scan_shape &s, const ScanPlan &plan);
void scan_set_carry(ScanArgs &a, const sn_scan_shape &s, const ScanPlan &p, void *ws);
hipError_t launch_scan_states(ScanArgs a, const sn_scan_shape &s, const ScanPlan &p, int wide, hipStream_t st);   // a.states from the inputs
hipError_t launch_scan_carry(const ScanArgs &a, const ScanPlan &p, bool reverse, hipStream_t st);

template <typename F> hipError_t by_lanes(int NL, F f)
{
    return NL == 2 ? f(SeqInt<2>()) : NL == 4 ? f(SeqInt<4>()) : NL == 8 ? f(SeqInt<8>()) : f(SeqInt<16>());
}
// f(lanes of a channel, width): with eight lanes and more a thread stages two channels at most, and twos are whole pieces
template <typename F> hipError_t by_lanes_and_width(int NL, int wide, F f)
{
    return by_lanes(NL, [&](auto L) {
        if (wide == 2) return f(L, SeqInt<2>());
        if constexpr (L.value < 8)
            if (wide == 1) return f(L, SeqInt<1>());
        return f(L, SeqInt<0>());
    });
}

}  // namespace sn
