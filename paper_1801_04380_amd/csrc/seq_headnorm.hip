// RMS norm of every head of queries and keys with the position rotation in the same pass, and its gradients.
//
// A dozen operations per element against two (backward: three) tensors read and written: bound by HBM.  A lane holds `unit`s of 2 E
// elements: the E pairs (i, i + rot/2) or (2i, 2i+1) of neighbouring angles, both halves in the same lane, so that the rotation exchanges
// nothing; behind rot_dim a unit is 2 E neighbours that are not turned.  LPH lanes (a power of two) hold a head, a wave 64 / LPH
// heads of one row at a time, NU units a lane.  The wave then takes the row's next heads, q's and k's in one list, loading the next ones
// before it works on these.  A row's angles are formed once, one by each lane, in 64 bits, and handed round through LDS.
#include "seq.h"

namespace sn {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;

struct HeadArgs {
    int rows, q_heads, heads, head_dim, rot_dim, interleaved, has_wq, has_wk;
    float eps;
};

template <typename T, int E> struct Raw {   // a unit as it lies in memory
    Pack<T, E> lo, hi;
    __device__ void zero()
    {
        lo.zero();
        hi.zero();
    }
    __device__ void load(const T *head, int pa, int pb, int nb, bool pairs)
    {
        lo.load(head + pa, E, true);
        if (pairs) hi.load(head + pa + E, E, true);
        else if (nb) hi.load(head + pb, E, true);
        else hi.zero();
    }
};

template <typename T, int E> struct Unit {
    float a[E], b[E];
    __device__ Unit() {}
    __device__ Unit(const Raw<T, E> &r, bool pairs)
    {
#pragma unroll
        for (int i = 0; i < E; ++i) {   // pairs: a, b alternate through the 2 E neighbours
            const float ea = 2 * i < E ? r.lo.get(2 * i < E ? 2 * i : 0) : r.hi.get(2 * i < E ? 0 : 2 * i - E);
            const float eb = 2 * i + 1 < E ? r.lo.get(2 * i + 1 < E ? 2 * i + 1 : 0) : r.hi.get(2 * i + 1 < E ? 0 : 2 * i + 1 - E);
            a[i] = pairs ? ea : r.lo.get(i);
            b[i] = pairs ? eb : r.hi.get(i);
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
            lo.store(head + pa, E, true);
            hi.store(head + pa + E, E, true);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                lo.set(i, a[i]);
                hi.set(i, b[i]);
            }
            lo.store(head + pa, E, true);
            if (nb) hi.store(head + pb, E, true);
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

// cos and sin of position * freq: the product and its remainder by whole turns in 64 bits
__device__ inline void turn_of(int position, float freq, float &c, float &s)
{
    const double turns = (double)position * (double)freq * 0.15915494309189533577;
    const float part = (float)(turns - rint(turns));
    sincospif(2.f * part, &s, &c);
}

template <int LPH> __device__ inline float head_sum(float v)
{
#pragma unroll
    for (int m = LPH / 2; m >= 1; m /= 2) v += __shfl_xor(v, m, 64);
    return v;
}

template <typename T, int E, int NU, int LPH, bool BWD>
__global__ void __launch_bounds__(THREADS) headnorm_kernel(const T *q, const T *k, const float *__restrict__ wq, const float *__restrict__ wk,
                                                           const int32_t *__restrict__ positions, const float *__restrict__ freq, const T *gq, const T *gk,
                                                           T *oq, T *ok, float *__restrict__ part, HeadArgs h, int64_t ld_q, int64_t ld_k, int64_t ld_gq,
                                                           int64_t ld_gk, int64_t ld_oq, int64_t ld_ok)
{
    constexpr int HPW = 64 / LPH;
    __shared__ float turn[WAVES][2][SN_HEADNORM_MAX_DIM / 2];   // of the wave's row
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, group = lane / LPH, l = lane % LPH;
    const int parts = gridDim.y;                       // the list of heads is cut into so many parts
    const int per = ((h.heads + HPW - 1) / HPW + parts - 1) / parts * HPW;
    const int h0 = blockIdx.y * per, h1 = min(h.heads, h0 + per), stride = gridDim.x * WAVES;
    float dw[2][BWD ? NU : 1][BWD ? E : 1][2] = {};

    const auto pick = [&](const T *pq, const T *pk, int64_t lq, int64_t lk, int row, int head) {
        return head < h.q_heads ? pq + (int64_t)row * lq + (int64_t)head * h.head_dim : pk + (int64_t)row * lk + (int64_t)(head - h.q_heads) * h.head_dim;
    };
    Raw<T, E> rx[NU], rg[BWD ? NU : 1];
    const auto fetch = [&](int row, int head) {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const Place<E> p(u * LPH + l, h);
            if (row < h.rows && head < h1 && p.there) {
                rx[u].load(pick(q, k, ld_q, ld_k, row, head), p.pa, p.pb, p.nb, p.pairs);
                if (BWD) rg[u].load(pick(gq, gk, ld_gq, ld_gk, row, head), p.pa, p.pb, p.nb, p.pairs);
            } else {
                rx[u].zero();
                if (BWD) rg[u].zero();
            }
        }
    };
    int row = blockIdx.x * WAVES + wave;
    fetch(row, h0 + group);
    for (; row < h.rows; row += stride) {
        const int pos = positions ? positions[row] : row;
        for (int i = lane; i < h.rot_dim / 2; i += 64) {
            float c, s;
            turn_of(pos, freq[i], c, s);
            turn[wave][0][i] = c;
            turn[wave][1][i] = s;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // a wave's own writes, read by its other lanes
        float co[NU][E], si[NU][E];
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const Place<E> p(u * LPH + l, h);
            const bool turned = p.there && p.angle >= 0;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                co[u][i] = turned ? turn[wave][0][turned ? p.angle + i : 0] : 1.f;
                si[u][i] = turned ? turn[wave][1][turned ? p.angle + i : 0] : 0.f;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before the next row's are written
        for (int head = h0 + group; head < h1 + group; head += HPW) {   // every lane goes round as often
            const bool here = head < h1, is_q = head < h.q_heads;
            T *o = (is_q ? oq + (int64_t)row * ld_oq + (int64_t)head * h.head_dim : ok + (int64_t)row * ld_ok + (int64_t)(head - h.q_heads) * h.head_dim);
            const float *w = is_q ? (h.has_wq ? wq : nullptr) : (h.has_wk ? wk : nullptr);
            Unit<T, E> v[NU], d[BWD ? NU : 1];
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const Place<E> p(u * LPH + l, h);
                v[u] = Unit<T, E>(rx[u], p.pairs);
                if (BWD) d[u] = Unit<T, E>(rg[u], p.pairs);
#pragma unroll
                for (int i = 0; i < E; ++i) sum = fmaf(v[u].a[i], v[u].a[i], fmaf(v[u].b[i], v[u].b[i], sum));
            }
            const bool more = head - group + HPW < h1;
            fetch(more ? row : row + stride, more ? head + HPW : h0 + group);
            const float r = 1.f / sqrtf(head_sum<LPH>(sum) / (float)h.head_dim + h.eps);
            if (!BWD) {
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const Place<E> p(u * LPH + l, h);
                    if (!here || !p.there) continue;
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        const float na = v[u].a[i] * r * (w ? w[p.at_a(i)] : 1.f), nb = v[u].b[i] * r * (w && p.nb ? w[p.at_b(i)] : 1.f);
                        v[u].a[i] = na * co[u][i] - nb * si[u][i];
                        v[u].b[i] = nb * co[u][i] + na * si[u][i];
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
                        const float ga = d[u].a[i] * co[u][i] + d[u].b[i] * si[u][i], gb = d[u].b[i] * co[u][i] - d[u].a[i] * si[u][i];
                        const float xa = v[u].a[i] * r, xb = v[u].b[i] * r;
                        dw[0][u][i][0] += is_q ? ga * xa : 0.f;
                        dw[0][u][i][1] += is_q ? gb * xb : 0.f;
                        dw[1][u][i][0] += is_q ? 0.f : ga * xa;
                        dw[1][u][i][1] += is_q ? 0.f : gb * xb;
                        d[u].a[i] = ga * (w && p.there ? w[p.at_a(i)] : 1.f);
                        d[u].b[i] = gb * (w && p.there && p.nb ? w[p.at_b(i)] : 1.f);
                        dot = fmaf(d[u].a[i], xa, fmaf(d[u].b[i], xb, dot));
                    }
                }
                dot = head_sum<LPH>(dot) / (float)h.head_dim;
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const Place<E> p(u * LPH + l, h);
                    if (!here || !p.there) continue;
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        d[u].a[i] = r * (d[u].a[i] - v[u].a[i] * r * dot);
                        d[u].b[i] = r * (d[u].b[i] - v[u].b[i] * r * dot);
                    }
                    d[u].store(o, p.pa, p.pb, p.nb, p.pairs);
                }
            }
        }
    }
    if (!BWD) return;
    // the workgroup's sums for both weights: over the head groups of a wave, then over its waves
    __shared__ float sums[WAVES][2][SN_HEADNORM_MAX_DIM];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const Place<E> p(u * LPH + l, h);
#pragma unroll
            for (int i = 0; i < E; ++i)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float s = dw[m][BWD ? u : 0][BWD ? i : 0][half];
#pragma unroll
                    for (int x = LPH; x < 64; x *= 2) s += __shfl_xor(s, x, 64);
                    if (group == 0 && p.there && (half == 0 || p.nb)) sums[wave][m][half ? p.at_b(i) : p.at_a(i)] = s;
                }
        }
    __syncthreads();
    float *to = part + (size_t)(blockIdx.y * gridDim.x + blockIdx.x) * 2 * h.head_dim;
    for (int i = threadIdx.x; i < 2 * h.head_dim; i += THREADS) {
        const int m = i >= h.head_dim, e = m ? i - h.head_dim : i;
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) s += sums[v][m][e];
        to[i] = s;
    }
}

// One workgroup per 16 elements of the two weights' gradients: 64 threads along the workgroups' sums, joined in a fixed order.
__global__ void __launch_bounds__(1024) headnorm_sum_kernel(const float *__restrict__ part, float *__restrict__ dwq, float *__restrict__ dwk, int head_dim, int parts)
{
    const int e = threadIdx.x % 16, lane = threadIdx.x / 16, i = blockIdx.x * 16 + e;
    __shared__ float sums[64][16];
    float s = 0.f;
    if (i < 2 * head_dim)
#pragma unroll 8
        for (int p = lane; p < parts; p += 64) s += part[(size_t)p * 2 * head_dim + i];
    sums[lane][e] = s;
    __syncthreads();
    if (lane || i >= 2 * head_dim) return;
    s = 0.f;
#pragma unroll
    for (int j = 0; j < 64; ++j) s += sums[j][e];
    if (i < head_dim) {
        if (dwq) dwq[i] = s;
    } else if (dwk) {
        dwk[i - head_dim] = s;
    }
}

// How many workgroups walk the rows, and into how many parts the list of heads is cut: waves for the chip where rows are few.
void grid_of(int64_t rows, int heads, dim3 *grid)
{
    int64_t blocks = (rows + WAVES - 1) / WAVES, most = 1024;
    if (blocks > most) blocks = most;
    if (blocks < 1) blocks = 1;
    int64_t parts = 1024 / blocks;
    if (parts > heads) parts = heads;
    if (parts < 1) parts = 1;
    *grid = dim3((unsigned)blocks, (unsigned)parts);
}

template <int V> struct Is { static constexpr int value = V; };

// f(E, NU, LPH): the widest unit that the sizes and the alignment allow
template <typename T, typename F> hipError_t by_size(int head_dim, int rot_dim, int aligned, F f)
{
    constexpr int most = 16 / (int)sizeof(T);
    int e = most;
    while (e > 1 && (e > aligned || (rot_dim / 2) % e || (head_dim - rot_dim) % e)) e /= 2;
    const int units = rot_dim / 2 / e + (head_dim - rot_dim + 2 * e - 1) / (2 * e);
    const auto pick = [&](auto E) {
        if (units <= 1) return f(E, Is<1>(), Is<1>());
        if (units <= 2) return f(E, Is<1>(), Is<2>());
        if (units <= 4) return f(E, Is<1>(), Is<4>());
        if (units <= 8) return f(E, Is<1>(), Is<8>());
        if (units <= 16) return f(E, Is<1>(), Is<16>());
        if (units <= 32) return f(E, Is<1>(), Is<32>());
        if (units <= 64) return f(E, Is<1>(), Is<64>());
        return f(E, Is<4>(), Is<64>());   // SN_HEADNORM_MAX_DIM / 2 units of one pair at most
    };
    if (e == 8) return pick(Is<most>());
    if (e == 4) return pick(Is<4>());
    if (e == 2) return pick(Is<2>());
    return pick(Is<1>());
}

int alignment(const void *p, int64_t ld, int esize)
{
    int v = 16 / esize;
    while (v > 1 && !rows_aligned(p, ld, esize, v)) v /= 2;
    return v;
}

HeadArgs args_of(const sn_headnorm_shape &s, const float *wq, const float *wk)
{
    return {(int)s.rows, s.q_heads, s.q_heads + s.k_heads, s.head_dim, s.rot_dim, s.interleaved, wq != nullptr, wk != nullptr, s.eps};
}

int least(int a, int b) { return a < b ? a : b; }

template <typename T, bool BWD>
hipError_t launch(const void *q, const void *k, const float *wq, const float *wk, const int32_t *pos, const float *freq, const void *gq, const void *gk, void *oq,
                  void *ok, int64_t ld_gq, int64_t ld_gk, int64_t ld_oq, int64_t ld_ok, const sn_headnorm_shape &s, float *part, hipStream_t st)
{
    int al = least(alignment(q, s.ld_q, sizeof(T)), alignment(oq, ld_oq, sizeof(T)));
    if (BWD) al = least(al, alignment(gq, ld_gq, sizeof(T)));
    if (s.k_heads) {
        al = least(al, least(alignment(k, s.ld_k, sizeof(T)), alignment(ok, ld_ok, sizeof(T))));
        if (BWD) al = least(al, alignment(gk, ld_gk, sizeof(T)));
    }
    while (s.head_dim % al) al /= 2;
    dim3 grid;
    grid_of(s.rows, s.q_heads + s.k_heads, &grid);
    return by_size<T>(s.head_dim, s.rot_dim, al, [&](auto E, auto NU, auto LPH) {
        headnorm_kernel<T, E.value, NU.value, LPH.value, BWD><<<grid, THREADS, 0, st>>>((const T *)q, (const T *)k, wq, wk, pos, freq, (const T *)gq, (const T *)gk, (T *)oq,
                                                                                        (T *)ok, part, args_of(s, wq, wk), s.ld_q, s.ld_k, ld_gq, ld_gk, ld_oq, ld_ok);
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
    dim3 grid;
    grid_of(rows, q_heads + k_heads, &grid);
    return align_up((size_t)grid.x * grid.y * 2 * head_dim * 4, 256);
}

hipError_t launch_headnorm_bwd(const void *q, const void *k, const float *wq, const float *wk, const int32_t *pos, const float *freq, const void *dyq,
                               const void *dyk, void *dq, void *dk, float *dwq, float *dwk, const sn_headnorm_shape &s, void *scratch, hipStream_t st)
{
    hipError_t e = s.dtype == SN_BF16
        ? launch<bf16_t, true>(q, k, wq, wk, pos, freq, dyq, dyk, dq, dk, s.ld_yq, s.ld_yk, s.ld_dq, s.ld_dk, s, (float *)scratch, st)
        : launch<float, true>(q, k, wq, wk, pos, freq, dyq, dyk, dq, dk, s.ld_yq, s.ld_yk, s.ld_dq, s.ld_dk, s, (float *)scratch, st);
    if (e != hipSuccess || (!dwq && !dwk)) return e;
    dim3 grid;
    grid_of(s.rows, s.q_heads + s.k_heads, &grid);
    headnorm_sum_kernel<<<(2 * s.head_dim + 15) / 16, 1024, 0, st>>>((const float *)scratch, dwq, dwk, s.head_dim, (int)(grid.x * grid.y));
    return hipGetLastError();
}

}  // namespace sn
