// RMS norm of every head of queries and keys with the position rotation in the same pass, and its gradients.
//
// A dozen operations per element against two (backward: three) tensors read and written: bound by HBM.  A lane holds `unit`s of 2 E
// elements: the E pairs (i, i + rot/2) or (2i, 2i+1) of neighbouring angles, both halves in the same lane, so that the rotation exchanges
// nothing; behind rot_dim a unit is 2 E neighbours that are not turned.  LPH lanes (a power of two) hold a head, a wave 64 / LPH
// heads of one row at a time, NU units a lane.  The wave then takes the row's next heads, loading them before it works on these.  A workgroup
// has to do with q or with k alone, whose weight its lanes hold.  A row's angles are formed once, one by each lane, in 64 bits, and handed
// round through LDS.  16384 rows, 32 and 8 heads of 128, bf16: forward 60 us (5.6 TB/s, part of it from the memory-side cache), backward
// 108 us (4.7 TB/s); 32 rows, 16 and 4 heads of 64: 4.2 us.
#include "seq.h"
#include <type_traits>

namespace sn {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;

struct HeadSide {   // q or k
    const void *x, *g;
    void *out;
    const float *w;
    int64_t ld_x, ld_g, ld_out;
    int heads, parts;   // its list of heads is cut into so many parts
};
struct HeadArgs {
    HeadSide side[2];
    const int32_t *positions;
    const float *freq;
    float *part;
    int rows, head_dim, rot_dim, interleaved;
    float eps;
};

template <typename T, int E> struct Raw {   // a unit as it lies in memory
    Pack<T, E> lo, hi;
    __device__ void load(const T *head, int pa, int pb)
    {
        lo.load(head + pa);
        hi.load(head + pb);
    }
};

template <typename T, int E> struct Unit {
    float a[E], b[E];
    __device__ Unit() {}
    // has_a, has_b: whether the halves are there
    __device__ Unit(const Raw<T, E> &r, bool pairs, bool has_a, bool has_b)
    {
#pragma unroll
        for (int i = 0; i < E; ++i) {   // pairs: a, b alternate through the 2 E neighbours
            const float ea = 2 * i < E ? r.lo.get(2 * i < E ? 2 * i : 0) : r.hi.get(2 * i < E ? 0 : 2 * i - E);
            const float eb = 2 * i + 1 < E ? r.lo.get(2 * i + 1 < E ? 2 * i + 1 : 0) : r.hi.get(2 * i + 1 < E ? 0 : 2 * i + 1 - E);
            a[i] = !has_a ? 0.f : pairs ? ea : r.lo.get(i);
            b[i] = !has_b ? 0.f : pairs ? eb : r.hi.get(i);
        }
    }
    __device__ void store(T *head, int pa, int pb, int nb, bool pairs) const
    {
        Pack<T, E> lo, hi;
        if (pairs) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (2 * i < E) lo.set(2 * i < E ? 2 * i : 0, a[i]); else hi.set(2 * i < E ? 0 : 2 * i - E, a[i]);
                if (2 * i + 1 < E) lo.set(2 * i + 1 < E ? 2 * i + 1 : 0, b[i]); else hi.set(2 * i + 1 < E ? 0 : 2 * i + 1 - E, b[i]);
            }
            lo.store(head + pa);
            hi.store(head + pa + E);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                lo.set(i, a[i]);
                hi.set(i, b[i]);
            }
            lo.store(head + pa);
            if (nb) hi.store(head + pb);
        }
    }
};

// Where unit u of a head lies: its halves' first elements (pairs: the first of 2 E neighbours), its first angle (-1: not turned).
template <int E> struct Place {
    int pa, pb, nb, angle;
    bool there, pairs;
    __device__ Place(int u, const HeadArgs &h)
    {
        const int turned = h.rot_dim / 2 / E;
        pairs = false;
        if (u < turned) {
            there = true;
            angle = u * E;
            pairs = h.interleaved;
            pa = pairs ? 2 * u * E : u * E;
            pb = h.rot_dim / 2 + u * E;
            nb = E;
        } else {
            pa = h.rot_dim + (u - turned) * 2 * E;
            pb = pa + E;
            there = pa < h.head_dim;
            nb = pb < h.head_dim ? E : 0;
            angle = -1;
        }
    }
    // the place of a's and b's element i in the head
    __device__ int at_a(int i) const { return pairs ? pa + 2 * i : pa + i; }
    __device__ int at_b(int i) const { return pairs ? pa + 2 * i + 1 : pb + i; }
};

// cos and sin of position * freq.  The product of the 31 and 24 bits, and that by 1 / (2 pi), are carried in two doubles each: the fraction of a turn
// is good to 2^-50 for angles up to 2^50, at far positions and high frequencies alike.  It is rounded to 24 bits because that is what sine and cosine
// take in 32 bits, and what the rounding took, below 2^-25 of a turn, is put back to first order: sin(a + d) = sin a + d cos a.
__device__ inline void turn_of(int position, float freq, float &c, float &s)
{
#pragma clang fp contract(off)   // each product by itself: what it lost is added by the line after it
    constexpr double turn = 0.15915494309189535, turn_lo = -9.839338337591243e-18;   // 1 / (2 pi)
    const double p = (double)position, f = (double)freq, angle = p * f, turns = angle * turn;
    const double lost = fma(angle, turn, -turns) + (angle * turn_lo + fma(p, f, -angle) * turn);
    const double part = (turns - rint(turns)) + lost, left = part - rint(part);
    const float near = (float)left, rest = (float)(left - (double)near) * 6.28318530717958647692f;
    float c0, s0;
    sincospif(2.f * near, &s0, &c0);
    c = fmaf(-s0, rest, c0);
    s = fmaf(c0, rest, s0);
}

// The sum over the LPH lanes of a head, in each of them.  Within 16 lanes by the cross-lane operands of the addition: neighbours, pairs,
// the mirror of four (whose four hold the same by then), eight apart.
template <int LPH> __device__ inline float head_sum(float v)
{
    const auto other = [](float x, auto how) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), how.value, 0xf, 0xf, true)); };
    if constexpr (LPH >= 2) v += other(v, std::integral_constant<int, 0xb1>());    // quad_perm:[1,0,3,2]
    if constexpr (LPH >= 4) v += other(v, std::integral_constant<int, 0x4e>());    // quad_perm:[2,3,0,1]
    if constexpr (LPH >= 8) v += other(v, std::integral_constant<int, 0x141>());   // row_half_mirror
    if constexpr (LPH >= 16) v += other(v, std::integral_constant<int, 0x128>());  // row_ror:8
    if constexpr (LPH >= 32) v += __shfl_xor(v, 16, 64);
    if constexpr (LPH >= 64) v += __shfl_xor(v, 32, 64);
    return v;
}

// 1 / sqrt(v) within one unit of the last place.  The instruction takes numbers below 2^-126 for zero: they are scaled, by a power of four.
__device__ inline float inv_root(float v)
{
    const bool small = v < 0x1p-126f;
    const float r = __builtin_amdgcn_rsqf(small ? v * 0x1p64f : v);
    return small ? r * 0x1p32f : r;
}

template <typename T, int E, int NU, int LPH, bool BWD>
__global__ void __launch_bounds__(THREADS) headnorm_kernel(HeadArgs h)
{
    constexpr int HPW = 64 / LPH;
    __shared__ float turn[WAVES][2][SN_HEADNORM_MAX_DIM / 2];   // of the wave's row
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, group = lane / LPH, l = lane % LPH;
    const bool is_q = (int)blockIdx.y < h.side[0].parts;
    const HeadSide &s = h.side[is_q ? 0 : 1];
    const int part = blockIdx.y - (is_q ? 0 : h.side[0].parts);
    const int per = ((s.heads + HPW - 1) / HPW + s.parts - 1) / s.parts * HPW;
    const int h0 = part * per, h1 = min(s.heads, h0 + per), stride = gridDim.x * WAVES;
    const float inv_dim = 1.f / (float)h.head_dim;
    float wa[NU][E], wb[NU][E], dw[BWD ? NU : 1][BWD ? E : 1][2] = {};
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        const Place<E> p(u * LPH + l, h);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            wa[u][i] = s.w && p.there ? s.w[p.at_a(i)] : 1.f;
            wb[u][i] = s.w && p.there && p.nb ? s.w[p.at_b(i)] : 1.f;
        }
    }
    Raw<T, E> rx[NU], rg[BWD ? NU : 1];
    const auto fetch = [&](int row, int head) {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const Place<E> p(u * LPH + l, h);   // without a condition, see Pack: from the last row, the last head, its first elements
            const int pa = p.there ? p.pa : 0, pb = !p.there ? 0 : p.pairs ? p.pa + E : p.nb ? p.pb : 0;
            const int64_t t = min(row, h.rows - 1), at = (int64_t)min(head, h1 - 1) * h.head_dim;
            rx[u].load((const T *)s.x + t * s.ld_x + at, pa, pb);
            if (BWD) rg[u].load((const T *)s.g + t * s.ld_g + at, pa, pb);
        }
    };
    int row = blockIdx.x * WAVES + wave;
    if (h0 < h1 && h.rows) fetch(row, h0 + group);
    for (; row < h.rows && h0 < h1; row += stride) {
        const int pos = h.positions ? h.positions[row] : row;
        for (int i = lane; i < h.rot_dim / 2; i += 64) {
            float c, sn;
            turn_of(pos, h.freq[i], c, sn);
            turn[wave][0][i] = c;
            turn[wave][1][i] = sn;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // a wave's own writes, read by its other lanes
        float co[NU][E], si[NU][E];
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const Place<E> p(u * LPH + l, h);
            const bool turned = p.there && p.angle >= 0;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                co[u][i] = turn[wave][0][turned ? p.angle + i : 0];   // not used otherwise
                si[u][i] = turn[wave][1][turned ? p.angle + i : 0];
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before the next row's are written
        for (int hb = h0; hb < h1; hb += HPW) {
            const int head = hb + group;
            const bool here = head < h1;
            T *o = (T *)s.out + (int64_t)row * s.ld_out + (int64_t)head * h.head_dim;
            Unit<T, E> v[NU], d[BWD ? NU : 1];
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const Place<E> p(u * LPH + l, h);
                v[u] = Unit<T, E>(rx[u], p.pairs, p.there, p.there && p.nb);
                if (BWD) d[u] = Unit<T, E>(rg[u], p.pairs, here && p.there, here && p.there && p.nb);
#pragma unroll
                for (int i = 0; i < E; ++i) sum = fmaf(v[u].a[i], v[u].a[i], fmaf(v[u].b[i], v[u].b[i], sum));
            }
            const bool more = hb + HPW < h1;
            fetch(more ? row : row + stride, more ? head + HPW : h0 + group);
            const float r = inv_root(fmaf(head_sum<LPH>(sum), inv_dim, h.eps));
            if (!BWD) {
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const Place<E> p(u * LPH + l, h);
                    if (!here || !p.there) continue;
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        const float na = v[u].a[i] * r * wa[u][i], nb = v[u].b[i] * r * wb[u][i];
                        // what is not turned is left out by choice, not by a sine of 0: an infinity would come through as NaN
                        v[u].a[i] = p.angle < 0 ? na : na * co[u][i] - nb * si[u][i];
                        v[u].b[i] = p.angle < 0 ? nb : nb * co[u][i] + na * si[u][i];
                    }
                    v[u].store(o, p.pa, p.pb, p.nb, p.pairs);
                }
            } else {
                float dot = 0.f;
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const Place<E> p(u * LPH + l, h);
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        const float ga = p.angle < 0 ? d[u].a[i] : d[u].a[i] * co[u][i] + d[u].b[i] * si[u][i];
                        const float gb = p.angle < 0 ? d[u].b[i] : d[u].b[i] * co[u][i] - d[u].a[i] * si[u][i];
                        v[u].a[i] *= r;
                        v[u].b[i] *= r;
                        dw[u][i][0] = fmaf(ga, v[u].a[i], dw[u][i][0]);
                        dw[u][i][1] = fmaf(gb, v[u].b[i], dw[u][i][1]);
                        d[u].a[i] = ga * wa[u][i];
                        d[u].b[i] = gb * wb[u][i];
                        dot = fmaf(d[u].a[i], v[u].a[i], fmaf(d[u].b[i], v[u].b[i], dot));
                    }
                }
                dot = head_sum<LPH>(dot) * inv_dim;
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const Place<E> p(u * LPH + l, h);
                    if (!here || !p.there) continue;
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        d[u].a[i] = r * fmaf(-dot, v[u].a[i], d[u].a[i]);
                        d[u].b[i] = r * fmaf(-dot, v[u].b[i], d[u].b[i]);
                    }
                    d[u].store(o, p.pa, p.pb, p.nb, p.pairs);
                }
            }
        }
    }
    if (!BWD) return;
    // the workgroup's sums for its weight: over the head groups of a wave, then over its waves
    __shared__ float sums[BWD ? WAVES : 1][BWD ? SN_HEADNORM_MAX_DIM : 1];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        const Place<E> p(u * LPH + l, h);
#pragma unroll
        for (int i = 0; i < E; ++i)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float v = dw[BWD ? u : 0][BWD ? i : 0][half];
#pragma unroll
                for (int x = LPH; x < 64; x *= 2) v += __shfl_xor(v, x, 64);
                if (group == 0 && p.there && (half == 0 || p.nb)) sums[BWD ? wave : 0][half ? p.at_b(i) : p.at_a(i)] = v;
            }
    }
    __syncthreads();
    float *to = h.part + (size_t)(blockIdx.y * gridDim.x + blockIdx.x) * h.head_dim;
    for (int i = threadIdx.x; i < h.head_dim; i += THREADS) {
        float v = 0.f;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) v += sums[BWD ? x : 0][i];
        to[i] = v;
    }
}

// One workgroup per 16 elements of a weight's gradient, y = 0 q's: 64 threads along the workgroups' sums, joined in a fixed order.
__global__ void __launch_bounds__(1024) headnorm_sum_kernel(const float *__restrict__ part, float *__restrict__ dwq, float *__restrict__ dwk, int head_dim, int q_parts,
                                                            int k_parts)
{
    const int e = threadIdx.x % 16, lane = threadIdx.x / 16, i = blockIdx.x * 16 + e, first = blockIdx.y ? q_parts : 0, count = blockIdx.y ? k_parts : q_parts;
    __shared__ float sums[64][16];
    LongSum s, all;
    if (i < head_dim)
#pragma unroll 8
        for (int p = lane; p < count; p += 64) s.add(part[(size_t)(first + p) * head_dim + i]);
    sums[lane][e] = s.total();
    __syncthreads();
    float *to = blockIdx.y ? dwk : dwq;
    if (lane || i >= head_dim || !to) return;
#pragma unroll
    for (int j = 0; j < 64; ++j) all.add(sums[j][e]);
    to[i] = all.total();
}

// How many workgroups walk the rows, and into how many parts the lists of heads are cut: waves for the chip where rows are few.  Backward (sums): as many more as
// it takes for a lane to add up 256 terms of a weight's gradient at most (a running sum is off by up to 2^-24 of the terms for each: over 2^25 equal rows in 1024
// workgroups 9e-5); the workgroups' sums are joined without loss.
struct HeadGrid {
    int blocks, q_parts, k_parts;
};
HeadGrid grid_of(int64_t rows, int q_heads, int k_heads, bool sums)
{
    constexpr int64_t TERMS = 256;
    HeadGrid g;
    const int64_t most = (rows + WAVES - 1) / WAVES, heads = q_heads > k_heads ? q_heads : k_heads;
    int64_t blocks = most > 1024 ? 1024 : most < 1 ? 1 : most, parts = 1024 / blocks;
    if (sums) {
        if (heads > parts * TERMS) parts = (heads + TERMS - 1) / TERMS;
        const int64_t terms = (heads + parts - 1) / parts, of_rows = TERMS / terms, enough = (most + of_rows - 1) / of_rows;   // TERMS / terms rows a wave
        if (enough > blocks) blocks = enough > 1 << 22 ? 1 << 22 : enough;
    }
    g.blocks = (int)blocks;
    g.q_parts = (int)(parts < q_heads ? parts : q_heads);
    g.k_parts = (int)(parts < k_heads ? parts : k_heads);
    return g;
}

// f(E, NU, LPH): the widest unit that the sizes allow, or a narrower one where a row's heads would leave half of a wave's lanes without work
// (4099 rows, 8 and 8 heads of 16 in fp32, us forward and backward: units of 8 elements 7.8, 12.9, of 2 6.5, 7.9)
template <typename T, typename F> hipError_t by_size(int head_dim, int rot_dim, int heads, F f)
{
    constexpr int most = 16 / (int)sizeof(T);
    int e = most;
    const auto units_of = [&](int e) { return rot_dim / 2 / e + (head_dim - rot_dim + 2 * e - 1) / (2 * e); };
    while (e > 1 && ((rot_dim / 2) % e || (head_dim - rot_dim) % e || heads * units_of(e) <= 32)) e /= 2;
    const int units = units_of(e);
    const auto pick = [&](auto E) {
        if (units <= 1) return f(E, SeqInt<1>(), SeqInt<1>());
        if (units <= 2) return f(E, SeqInt<1>(), SeqInt<2>());
        if (units <= 4) return f(E, SeqInt<1>(), SeqInt<4>());
        if (units <= 8) return f(E, SeqInt<1>(), SeqInt<8>());
        if (units <= 16) return f(E, SeqInt<1>(), SeqInt<16>());
        constexpr int largest = SN_HEADNORM_MAX_DIM / 2 / E.value;   // units that there can be
        if constexpr (largest > 32)
            if (units > 32) {
                if constexpr (largest > 64)
                    if (units > 64) return f(E, SeqInt<largest / 64>(), SeqInt<64>());
                return f(E, SeqInt<1>(), SeqInt<64>());
            }
        return f(E, SeqInt<1>(), SeqInt<32>());
    };
    if (e == 8) return pick(SeqInt<most>());
    if (e == 4) return pick(SeqInt<4>());
    if (e == 2) return pick(SeqInt<2>());
    return pick(SeqInt<1>());
}

template <typename T, bool BWD>
hipError_t launch(const void *q, const void *k, const float *wq, const float *wk, const int32_t *pos, const float *freq, const void *gq, const void *gk, void *oq,
                  void *ok, int64_t ld_gq, int64_t ld_gk, int64_t ld_oq, int64_t ld_ok, const sn_headnorm_shape &s, float *part, hipStream_t st)
{
    const HeadGrid g = grid_of(s.rows, s.q_heads, s.k_heads, BWD);
    const HeadArgs h = {{{q, gq, oq, wq, s.ld_q, ld_gq, ld_oq, s.q_heads, g.q_parts}, {k, gk, ok, wk, s.ld_k, ld_gk, ld_ok, s.k_heads, g.k_parts}}, pos, freq, part,
                        (int)s.rows, s.head_dim, s.rot_dim, s.interleaved, s.eps};
    return by_size<T>(s.head_dim, s.rot_dim, s.q_heads > s.k_heads ? s.q_heads : s.k_heads, [&](auto E, auto NU, auto LPH) {
        headnorm_kernel<T, E.value, NU.value, LPH.value, BWD><<<dim3(g.blocks, g.q_parts + g.k_parts), THREADS, 0, st>>>(h);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_headnorm_fwd(const void *q, const void *k, const float *wq, const float *wk, const int32_t *pos, const float *freq, void *yq, void *yk,
                               const sn_headnorm_shape &s, hipStream_t st)
{
    return s.dtype == SN_BF16 ? launch<bf16_t, false>(q, k, wq, wk, pos, freq, nullptr, nullptr, yq, yk, 0, 0, s.ld_yq, s.ld_yk, s, nullptr, st)
                              : launch<float, false>(q, k, wq, wk, pos, freq, nullptr, nullptr, yq, yk, 0, 0, s.ld_yq, s.ld_yk, s, nullptr, st);
}

size_t headnorm_scratch_bytes(int64_t rows, int q_heads, int k_heads, int head_dim)
{
    const HeadGrid g = grid_of(rows, q_heads, k_heads, true);
    return align_up((size_t)g.blocks * (g.q_parts + g.k_parts) * head_dim * 4, 256);
}

hipError_t launch_headnorm_bwd(const void *q, const void *k, const float *wq, const float *wk, const int32_t *pos, const float *freq, const void *dyq,
                               const void *dyk, void *dq, void *dk, float *dwq, float *dwk, const sn_headnorm_shape &s, void *scratch, hipStream_t st)
{
    hipError_t e = s.dtype == SN_BF16
        ? launch<bf16_t, true>(q, k, wq, wk, pos, freq, dyq, dyk, dq, dk, s.ld_yq, s.ld_yk, s.ld_dq, s.ld_dk, s, (float *)scratch, st)
        : launch<float, true>(q, k, wq, wk, pos, freq, dyq, dyk, dq, dk, s.ld_yq, s.ld_yk, s.ld_dq, s.ld_dk, s, (float *)scratch, st);
    if (e != hipSuccess || (!dwq && !dwk)) return e;
    const HeadGrid g = grid_of(s.rows, s.q_heads, s.k_heads, true);
    headnorm_sum_kernel<<<dim3((s.head_dim + 15) / 16, 2), 1024, 0, st>>>((const float *)scratch, dwq, dwk, s.head_dim, g.blocks * g.q_parts, g.blocks * g.k_parts);
    return hipGetLastError();
}

}  // namespace sn
