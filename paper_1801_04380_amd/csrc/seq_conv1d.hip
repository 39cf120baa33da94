// The short causal convolution along the tokens (one filter of up to 8 taps per channel, bias and SiLU in the same pass).
//
// Two operations per tap and a sigmoid per element against two (backward: three) tensors read and written: bound by HBM.  A thread owns V
// neighbouring channels (16 bytes if there are as many; the last thread's are moved back to end with the row, and what it has in common with
// the thread before it is computed and written twice alike) and walks down a run of rows with the taps' inputs in registers, so that an
// input row is loaded once but for the width - 1 rows in front of the run.  16384 x 4096, four taps, bf16: forward 57 us (4.7 TB/s),
// backward 100 us (4.0 TB/s); one token for four rows of 1024: 2.8 us, a launch's latency.
#include "seq.h"

namespace sn {
namespace {

constexpr int THREADS = 256;

// The filters and biases of V channels, taps innermost in memory.
template <typename T, int V, int W> struct Taps {
    float w[V][W], b[V];
    __device__ void load(const T *wp, const float *bp, int c)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            b[i] = bp ? bp[c + i] : 0.f;
#pragma unroll
            for (int j = 0; j < W; ++j) w[i][j] = seq_ld<T>(wp + (size_t)c * W + i * W + j);
        }
    }
    __device__ float p(int i, const Pack<T, V> *in) const   // of channel i from its W inputs
    {
        float v = b[i];
#pragma unroll
        for (int j = 0; j < W; ++j) v = fmaf(w[i][j], in[j].get(i), v);
        return v;
    }
};

template <typename T, int V> __device__ inline void load_each(Pack<T, V> &v, const T *p)
{
#pragma unroll
    for (int i = 0; i < V; ++i) v.e[i] = p[i];
}
template <typename T, int V> __device__ inline void store_each(const Pack<T, V> &v, T *p)
{
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = v.e[i];
}

// The input under a tap: row src of x where the sequence that begins at `begin` holds it, a row of the initial state in front of it.
template <typename T, int V>
__device__ inline Pack<T, V> tap_input(const T *x, int64_t ld, const T *state, int channels, int W, const SeqAt &at, int src, int c)
{
    Pack<T, V> v;
    if (src >= at.begin) v.load(x + (int64_t)src * ld + c);
    else if (state) load_each(v, state + ((int64_t)at.s * (W - 1) + (W - 1 + src - at.begin)) * channels + c);
    else v.zero();
    return v;
}

template <typename T, int V, int W>
__global__ void __launch_bounds__(THREADS) conv1d_fwd_kernel(const T *__restrict__ x, const T *__restrict__ w, const float *__restrict__ bias, T *__restrict__ y,
                                                             int channels, int silu, int64_t ld_x, int64_t ld_y, SeqRows rows, int run, int runs,
                                                             const T *__restrict__ state_in, T *__restrict__ state_out)
{
    constexpr int R = 8;   // rows at a time: their loads are all on their way before the first is used
    const bool mine = (blockIdx.x * THREADS + threadIdx.x) * V < channels;
    const int c = mine ? min((int)(blockIdx.x * THREADS + threadIdx.x) * V, channels - V) : 0;
    if ((int)blockIdx.y >= runs) {
        each_empty(rows, blockIdx.y - runs, gridDim.y - runs, [&](int s) {
            if (!mine) return;
            const int64_t k = (int64_t)s * (W - 1) * channels + c;
            Pack<T, V> v[W];   // all on their way before the first is stored
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
                if (state_in) v[j].load(state_in + k + (int64_t)j * channels);
                else v[j].zero();
#pragma unroll
            for (int j = 0; j < W - 1; ++j) v[j].store(state_out + k + (int64_t)j * channels);
        });
        return;
    }
    const int r0 = blockIdx.y * run, r1 = min(r0 + run, rows.rows);
    if (mine && r0 < r1) {
        Taps<T, V, W> taps;
        taps.load(w, bias, c);
        SeqAt at = seq_find(rows, r0);
        Pack<T, V> in[W - 1 + R], ahead[R];   // the rows in front, if the last turn was a whole one, and this turn's; the next turn's
        const auto fetch = [&](int b) {
#pragma unroll
            for (int k = 0; k < R; ++k) ahead[k].load(x + (int64_t)min(b + k, r1 - 1) * ld_x + c);
        };
        bool have = false;
        fetch(r0);
        for (int b = r0; b < r1; b += R) {
            seq_forward(rows, at, b);
#pragma unroll
            for (int k = 0; k < R; ++k) in[W - 1 + k] = ahead[k];
            fetch(b + R);
            if (at.holds(b, rows) && b - (W - 1) >= at.begin && b + R <= min(at.end, r1) && !(state_out && b + R == at.end)) {
                if (!have)
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) in[j].load(x + (int64_t)(b - (W - 1) + j) * ld_x + c);
                have = true;
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    Pack<T, V> out;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float p = taps.p(i, &in[k]);
                        out.set(i, silu ? p * sigmoid(p) : p);
                    }
                    out.store(y + (int64_t)(b + k) * ld_y + c);
                }
#pragma unroll
                for (int j = 0; j < W - 1; ++j) in[j] = in[R + j];
                continue;
            }
            // a sequence begins or ends here: row by row
            have = false;
            for (int t = b; t < min(b + R, r1); ++t) {
                seq_forward(rows, at, t);
                if (!at.holds(t, rows)) continue;
                Pack<T, V> tap[W], out;
#pragma unroll
                for (int j = 0; j < W; ++j) tap[j] = tap_input<T, V>(x, ld_x, state_in, channels, W, at, t - (W - 1) + j, c);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float p = taps.p(i, tap);
                    out.set(i, silu ? p * sigmoid(p) : p);
                }
                out.store(y + (int64_t)t * ld_y + c);
                if (state_out && t == at.end - 1)
#pragma unroll
                    for (int j = 1; j < W; ++j) store_each(tap[j], state_out + ((int64_t)at.s * (W - 1) + j - 1) * channels + c);
            }
        }
    }
}

// d y / d p
__device__ inline float silu_slope(float p)
{
    const float s = sigmoid(p);
    return s * (1.f + p * (1.f - s));
}

// part[slice][W + 1][channels]: the slice's sums for dw, then for dbias.
// A thread walks down the rows r0 .. r1 - 1 of its slice, R at a time.  A turn at b reads x and dy of the rows b + W - 1 .. b + R + W - 2,
// makes their dp, and with the W - 1 rows in front, which it has, dx of rows b .. b + R - 1.  The first turn, at r0 - R, only fills what the next
// one takes over; R >= 2 (W - 1) rows make that complete.
template <typename T, int V, int W>
__global__ void __launch_bounds__(THREADS) conv1d_bwd_kernel(const T *__restrict__ x, const T *__restrict__ w, const float *__restrict__ bias, const T *__restrict__ dy,
                                                             T *__restrict__ dx, float *__restrict__ part, int channels, int silu, int64_t ld_x, int64_t ld_y,
                                                             int64_t ld_dx, SeqRows rows, int run, const T *__restrict__ state_in,
                                                             const T *__restrict__ dstate_out)
{
    constexpr int R = W <= 5 ? 8 : 16, H = W - 1;
    const unsigned blocks = (channels + V * THREADS - 1) / (V * THREADS), slice = blockIdx.x / blocks, first = (blockIdx.x % blocks * THREADS + threadIdx.x) * V;
    if (first >= (unsigned)channels) return;
    const int c = min((int)first, channels - V);
    Taps<T, V, W> taps;
    taps.load(w, bias, c);
    const int r0 = slice * run, r1 = min(r0 + run, rows.rows);
    float dw[V][W] = {}, db[V] = {};
    if (r0 < r1) {
        float in[H + R][V] = {}, dp[H + R][V] = {};   // x and dp of rows b .. b + R + H - 1
        SeqAt lead = seq_find(rows, max(r0 - R + H, 0)), trail = seq_find(rows, r0);
        for (int b = r0 - R; b < r1; b += R) {
            Pack<T, V> xs[R], gs[R];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const int t = min(max(b + H + k, 0), rows.rows - 1);
                xs[k].load(x + (int64_t)t * ld_x + c);
                gs[k].load(dy + (int64_t)t * ld_y + c);
            }
            if (b >= r0) seq_forward(rows, trail, b);
            const bool plain = b >= r0 && b + H + R <= min(trail.end, r1) && trail.holds(b, rows);
#pragma unroll
            for (int k = 0; k < R; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) in[H + k][i] = xs[k].get(i);
            if (plain) {
#pragma unroll
                for (int k = 0; k < R; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float p = taps.b[i], d = gs[k].get(i);
                        if (silu) {
#pragma unroll
                            for (int j = 0; j < W; ++j) p = fmaf(taps.w[i][j], in[k + j][i], p);
                            d *= silu_slope(p);
                        }
                        dp[H + k][i] = d;
                        db[i] += d;
#pragma unroll
                        for (int j = 0; j < W; ++j) dw[i][j] = fmaf(d, in[k + j][i], dw[i][j]);
                    }
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    Pack<T, V> out;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float g = 0.f;
#pragma unroll
                        for (int j = 0; j < W; ++j) g = fmaf(taps.w[i][H - j], dp[k + j][i], g);
                        out.set(i, g);
                    }
                    out.store(dx + (int64_t)(b + k) * ld_dx + c);
                }
            } else {
                // the slice's or a sequence's first or last rows are among these
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    const int t = b + H + k;
                    const bool mine = t >= r0 && t < r1;
                    seq_forward(rows, lead, t);
                    const bool there = t >= 0 && lead.holds(t, rows);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float tap[W], p = taps.b[i], d = there ? gs[k].get(i) : 0.f;
#pragma unroll
                        for (int j = 0; j < W; ++j) {
                            const int src = t - H + j;
                            tap[j] = src >= lead.begin ? in[k + j][i] : 0.f;
                            if (there && src < lead.begin && state_in)
                                tap[j] = seq_ld<T>(state_in + ((int64_t)lead.s * H + H + src - lead.begin) * channels + c + i);
                            p = fmaf(taps.w[i][j], tap[j], p);
                        }
                        if (silu) d = there ? d * silu_slope(p) : 0.f;
                        dp[H + k][i] = d;
                        if (there && mine) {
                            db[i] += d;
#pragma unroll
                            for (int j = 0; j < W; ++j) dw[i][j] = fmaf(d, tap[j], dw[i][j]);
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    const int t = b + k;
                    if (t < r0 || t >= r1) continue;
                    seq_forward(rows, trail, t);
                    if (!trail.holds(t, rows)) continue;
                    Pack<T, V> out;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float g = 0.f;
#pragma unroll
                        for (int j = 0; j < W; ++j)
                            if (t + j < trail.end) g = fmaf(taps.w[i][H - j], dp[k + j][i], g);
                        if (dstate_out && t >= trail.end - H) g += seq_ld<T>(dstate_out + ((int64_t)trail.s * H + t - (trail.end - H)) * channels + c + i);
                        out.set(i, g);
                    }
                    out.store(dx + (int64_t)t * ld_dx + c);
                }
            }
#pragma unroll
            for (int j = 0; j < H; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    in[j][i] = in[R + j][i];
                    dp[j][i] = dp[R + j][i];
                }
        }
    }
    float *to = part + (size_t)slice * (W + 1) * channels + c;
#pragma unroll
    for (int j = 0; j <= W; ++j) {
        Pack<float, V> v;
#pragma unroll
        for (int i = 0; i < V; ++i) v.e[i] = j < W ? dw[i][j < W ? j : 0] : db[i];
        v.store(to + (size_t)j * channels);
    }
}

// The gradient of the initial states: one thread per sequence and channel.
template <typename T, int W>
__global__ void __launch_bounds__(THREADS) conv1d_dstate_kernel(const T *__restrict__ x, const T *__restrict__ w, const float *__restrict__ bias, const T *__restrict__ dy,
                                                                int channels, int silu, int64_t ld_x, int64_t ld_y, SeqRows rows, const T *__restrict__ state_in,
                                                                const T *__restrict__ dstate_out, T *__restrict__ dstate_in)
{
    const int c = blockIdx.y * THREADS + threadIdx.x, s = blockIdx.x;
    if (c >= channels) return;
    SeqAt at;
    if (rows.off) {
        at = seq_clamped(rows, s);
    } else {
        at.s = s; at.begin = s * rows.len; at.end = at.begin + rows.len;
    }
    const int len = max(at.end - at.begin, 0);
    Taps<T, 1, W> taps;
    taps.load(w, bias, c);
    float dp[W];  // of the sequence's first rows
#pragma unroll
    for (int e = 0; e < W - 1; ++e) {
        dp[e] = 0.f;
        if (e >= len) continue;
        const int t = at.begin + e;
        Pack<T, 1> in[W];
#pragma unroll
        for (int j = 0; j < W; ++j) in[j] = tap_input<T, 1>(x, ld_x, state_in, channels, W, at, t - (W - 1) + j, c);
        dp[e] = seq_ld<T>(dy + (int64_t)t * ld_y + c);
        if (silu) dp[e] *= silu_slope(taps.p(0, in));
    }
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {   // the state's row i stands W - 1 - i rows in front of the sequence
        float g = 0.f;
#pragma unroll
        for (int e = 0; e <= i; ++e) g = fmaf(taps.w[0][i - e], dp[e], g);   // it is tap i - e of row e
        const int left = i - len;       // its row in the final state
        if (dstate_out && left >= 0) g += seq_ld<T>(dstate_out + ((int64_t)s * (W - 1) + left) * channels + c);
        seq_st(dstate_in + ((int64_t)s * (W - 1) + i) * channels + c, g);
    }
}

// dw and dbias from the slices' sums: 16 threads along the slices of each value, joined in a fixed order.
__global__ void __launch_bounds__(THREADS) conv1d_sum_kernel(const float *__restrict__ part, float *__restrict__ dw, float *__restrict__ dbias, int channels, int width, int slices)
{
    __shared__ float sums[16][16];
    const int lane = threadIdx.x / 16, c = blockIdx.x * 16 + threadIdx.x % 16, j = blockIdx.y;
    LongSum sum, all;
    if (c < channels)
#pragma unroll 8
        for (int s = lane; s < slices; s += 16) sum.add(part[((size_t)s * (width + 1) + j) * channels + c]);
    sums[lane][threadIdx.x % 16] = sum.total();
    __syncthreads();
    if (lane || c >= channels) return;
#pragma unroll
    for (int s = 0; s < 16; ++s) all.add(sums[s][threadIdx.x]);
    if (j < width) dw[(size_t)c * width + j] = all.total();
    else if (dbias) dbias[c] = all.total();
}

template <typename T, int V, int W>
__global__ void __launch_bounds__(THREADS) conv1d_step_kernel(const T *__restrict__ x, const T *__restrict__ w, const float *__restrict__ bias, T *__restrict__ y,
                                                              const T *state, T *state_out, const int32_t *__restrict__ slots, int num_slots, int channels,
                                                              int silu, int64_t ld_x, int64_t ld_y)
{
    const int c = (blockIdx.y * THREADS + threadIdx.x) * V, row = blockIdx.x;
    if (c >= channels) return;
    const int slot = step_slot(slots, row, num_slots);
    if (slot < 0) return;
    Taps<T, V, W> taps;
    taps.load(w, bias, c);
    Pack<T, V> in[W], out;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) in[j].load(state + ((int64_t)slot * (W - 1) + j) * channels + c);
    in[W - 1].load(x + (int64_t)row * ld_x + c);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float p = taps.p(i, in);
        out.set(i, silu ? p * sigmoid(p) : p);
    }
    out.store(y + (int64_t)row * ld_y + c);
#pragma unroll
    for (int j = 1; j < W; ++j) in[j].store(state_out + ((int64_t)slot * (W - 1) + j - 1) * channels + c);
}

// f(type, width) with both as types
template <typename F> hipError_t by_width(int width, F f)
{
    switch (width) {
    case 1: return f(SeqInt<1>());
    case 2: return f(SeqInt<2>());
    case 3: return f(SeqInt<3>());
    case 4: return f(SeqInt<4>());
    case 5: return f(SeqInt<5>());
    case 6: return f(SeqInt<6>());
    case 7: return f(SeqInt<7>());
    default: return f(SeqInt<8>());
    }
}

SeqRows rows_of(const sn_conv1d_shape &s, const int32_t *off)
{
    return {off, s.seqs, (int)(s.rows / s.seqs), (int)s.rows};
}

// Rows of a workgroup's run, a multiple of 16: about 512 workgroups over `blocks` channel blocks, two waves a SIMD, each with eight rows' loads on their
// way; `least` rows at least, beside which the filters and the rows in front cost little: forward 16 (5003 x 1001 in fp32 12.8 us, with 32 14.8).
int run_of(int64_t rows, int blocks, int least)
{
    const int64_t want = (512 + blocks - 1) / blocks;
    const int64_t run = ((rows + want - 1) / want + 15) / 16 * 16;
    return (int)(run < least ? least : run);
}

// The channels of a thread: MOST if there are as many (IN_WHOLE: and no rest), else 1.
template <int MOST, bool IN_WHOLE, typename F> hipError_t by_vector(int channels, F f)
{
    if (channels >= MOST && !(IN_WHOLE && channels % MOST)) return f(SeqInt<MOST>());
    return f(SeqInt<1>());
}

template <typename T> hipError_t fwd(const void *x, const void *w, const float *bias, void *y, const sn_conv1d_shape &s, const int32_t *off, const void *state_in,
                                     void *state_out, hipStream_t st)
{
    return by_width(s.width, [&](auto W) {
        return by_vector<16 / sizeof(T), false>(s.channels, [&](auto V) {
            const SeqRows rows = rows_of(s, off);
            const int blocks = div_up(s.channels, V.value * THREADS), run = run_of(s.rows, blocks, 16), runs = div_up(s.rows, run);
            const int groups = runs + empty_groups(state_out && W.value > 1, rows);
            if (!groups) return hipSuccess;
            conv1d_fwd_kernel<T, V.value, W.value><<<dim3(blocks, groups), THREADS, 0, st>>>(
                (const T *)x, (const T *)w, bias, (T *)y, s.channels, s.silu, s.ld_x, s.ld_y, rows, run, runs, (const T *)state_in, (T *)state_out);
            return hipGetLastError();
        });
    });
}

constexpr int BWD_V = 4;   // channels of a thread at most: with 8 the windows of x and dp alone would take 176 registers

// 64 rows at least, so that the turn that fills the windows costs little, and 256 at most: the sums for dw and dbias are running sums over them, off by up to
// 2^-24 of the terms for each (over 2^24 equal rows in 512 runs 3e-4); the slices' sums are joined without loss.
int bwd_run(int64_t rows, int channels)
{
    const int run = run_of(rows, div_up(channels, BWD_V * THREADS), 64);
    return run > 256 ? 256 : run;
}

template <typename T> hipError_t bwd(const void *x, const void *w, const float *bias, const void *dy, void *dx, float *dw, float *dbias, const sn_conv1d_shape &s,
                                     const int32_t *off, const void *state_in, const void *dstate_out, void *dstate_in, void *scratch, hipStream_t st)
{
    return by_width(s.width, [&](auto W) {
        const int run = bwd_run(s.rows, s.channels), slices = s.rows ? div_up(s.rows, run) : 1;
        const SeqRows rows = rows_of(s, off);
        hipError_t e = by_vector<BWD_V, false>(s.channels, [&](auto V) {
            conv1d_bwd_kernel<T, V.value, W.value><<<(unsigned)div_up(s.channels, V.value * THREADS) * slices, THREADS, 0, st>>>(
                (const T *)x, (const T *)w, bias, (const T *)dy, (T *)dx, (float *)scratch, s.channels, s.silu, s.ld_x, s.ld_y, s.ld_dx, rows, run,
                (const T *)state_in, (const T *)dstate_out);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
        conv1d_sum_kernel<<<dim3(div_up(s.channels, 16), s.width + 1), THREADS, 0, st>>>((const float *)scratch, dw, dbias, s.channels, s.width, slices);
        e = hipGetLastError();
        if (e != hipSuccess || !dstate_in) return e;
        if constexpr (W.value > 1) {
            conv1d_dstate_kernel<T, W.value><<<dim3(s.seqs, div_up(s.channels, THREADS)), THREADS, 0, st>>>(
                (const T *)x, (const T *)w, bias, (const T *)dy, s.channels, s.silu, s.ld_x, s.ld_y, rows, (const T *)state_in, (const T *)dstate_out, (T *)dstate_in);
            e = hipGetLastError();
        }
        return e;
    });
}

template <typename T> hipError_t step(const void *x, const void *w, const float *bias, void *y, const void *state, void *state_out, const int32_t *slots, int num_slots,
                                      const sn_conv1d_shape &s, hipStream_t st)
{
    return by_width(s.width, [&](auto W) {
        // a state updated in place must not be read by two threads
        return by_vector<16 / sizeof(T), true>(s.channels, [&](auto V) {
            conv1d_step_kernel<T, V.value, W.value><<<dim3((int)s.rows, div_up(s.channels, V.value * THREADS)), THREADS, 0, st>>>(
                (const T *)x, (const T *)w, bias, (T *)y, (const T *)state, (T *)state_out, slots, num_slots, s.channels, s.silu, s.ld_x, s.ld_y);
            return hipGetLastError();
        });
    });
}

}  // namespace

hipError_t launch_conv1d_fwd(const void *x, const void *w, const float *bias, void *y, const sn_conv1d_shape &s, const int32_t *off, const void *state_in,
                             void *state_out, hipStream_t st)
{
    return s.dtype == SN_BF16 ? fwd<bf16_t>(x, w, bias, y, s, off, state_in, state_out, st) : fwd<float>(x, w, bias, y, s, off, state_in, state_out, st);
}

size_t conv1d_scratch_bytes(int64_t rows, int channels, int width)
{
    const int slices = rows ? div_up(rows, bwd_run(rows, channels)) : 1;
    return align_up((size_t)slices * (width + 1) * channels * 4, 256);
}

hipError_t launch_conv1d_bwd(const void *x, const void *w, const float *bias, const void *dy, void *dx, float *dw, float *dbias, const sn_conv1d_shape &s,
                             const int32_t *off, const void *state_in, const void *dstate_out, void *dstate_in, void *scratch, hipStream_t st)
{
    return s.dtype == SN_BF16 ? bwd<bf16_t>(x, w, bias, dy, dx, dw, dbias, s, off, state_in, dstate_out, dstate_in, scratch, st)
                              : bwd<float>(x, w, bias, dy, dx, dw, dbias, s, off, state_in, dstate_out, dstate_in, scratch, st);
}

hipError_t launch_conv1d_step(const void *x, const void *w, const float *bias, void *y, const void *state, void *state_out, const int32_t *slots, int num_slots,
                              const sn_conv1d_shape &s, hipStream_t st)
{
    return s.dtype == SN_BF16 ? step<bf16_t>(x, w, bias, y, state, state_out, slots, num_slots, s, st)
                              : step<float>(x, w, bias, y, state, state_out, slots, num_slots, s, st);
}

}  // namespace sn
