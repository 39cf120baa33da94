// What the kernels of the token-sequence layers share: element access at any alignment, exponentials, long sums.
#pragma once
#include "sn_internal.h"
#include "sn_seq.h"
#include "seq_walk.h"

namespace sn {

template <typename T> __device__ inline float seq_ld(const T *p);
template <> __device__ inline float seq_ld<float>(const float *p) { return *p; }
template <> __device__ inline float seq_ld<bf16_t>(const bf16_t *p) { return bf16_to_f32(*p); }
__device__ inline void seq_st(float *p, float v) { *p = v; }
__device__ inline void seq_st(bf16_t *p, float v) { *p = f32_to_bf16(v); }

// V neighbouring elements as they lie in memory, loaded and stored in one access, at an element's alignment: global memory takes them there.  What a lane has nothing to load
// from it loads from some other place and leaves out later: a load under a condition of the lane's own would be waited for right
// where the two ways meet, and nothing could be loaded ahead.
template <int BYTES> struct Word;
template <> struct Word<2> { typedef uint16_t type; };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Word<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <typename T, int V> struct alignas(sizeof(T) * V) Pack {
    typedef typename Word<sizeof(T) * V>::type W;   // the access, as one value: a copy of the elements would be split up and stored in parts
    struct __attribute__((packed, aligned(sizeof(T)))) At { W v; };
    T e[V];
    __device__ void zero()
    {
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = 0;
    }
    __device__ void load(const T *p) { *this = __builtin_bit_cast(Pack, reinterpret_cast<const At *>(p)->v); }
    __device__ void store(T *p) const { reinterpret_cast<At *>(p)->v = __builtin_bit_cast(W, *this); }
    __device__ float get(int i) const { return seq_ld<T>(&e[i]); }
    __device__ void set(int i, float v) { seq_st(&e[i], v); }
};

// The states of sequences without rows pass through: workgroups of their own, behind those that walk the rows, look at EMPTY_AT sequences at a time.  (One
// workgroup for all of them took 16.3 ms over 800 rows and 4094 empty sequences of 2048 channels, four taps; with these, and none of
// them walked one by one, the call takes 0.03.)  They are there only for calls that hand states on and may have such sequences.
constexpr int EMPTY_AT = 16;
inline int empty_groups(bool wanted, const SeqRows &r)
{
    const int groups = (r.seqs + EMPTY_AT - 1) / EMPTY_AT, most = 1 << 12;   // a grid's second dimension ends at 2^16
    return !wanted || (!r.off && r.rows) ? 0 : groups < most ? groups : most;
}
// f(s) for those that group `at` of `count` looks at, by all lanes of a wave together.
template <typename F> __device__ inline void each_empty(const SeqRows &r, int at, int count, F f)
{
    const int lane = threadIdx.x & 63;
    for (int s0 = at * EMPTY_AT; s0 < r.seqs; s0 += count * EMPTY_AT) {
        const int s = s0 + lane;
        uint64_t empty = __ballot(lane < EMPTY_AT && s < r.seqs && (!r.off || r.off[s] == r.off[s + 1]));
        for (; empty; empty &= empty - 1) f(s0 + __builtin_ctzll(empty));
    }
}

// The instructions for 2^x, log2 x and 1 / x, each within one unit of the last place; e^x and log through them.  For |x| up to 20 the product with
// log2(e) adds 20 * 2^-24 to the relative error of e^x.  2^x below 2^-126 is 0.
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float exp_fast(float x) { return exp2_fast(x * 1.44269504088896340736f); }
__device__ inline float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ inline float sigmoid(float x) { return rcp_fast(1.f + exp_fast(-x)); }

// log(1 + e^x).  With u = 1 + e^x as rounded, log(1 + e^x) = log(u) + (e^x - (u - 1)) / u to first order in what the rounding lost, and u - 1 is
// exact.  Below u = 4 the division is left out (what was lost is half a step of u at most, 2^-23: the result is off by less than 2^-23 * 3/4 of
// log(4), and by nothing to speak of near u = 1, where it counts); from there on the whole correction, below 2^-24 of a result above log(4).  From 20
// on log(1 + e^-x) is below half a step of x.
__device__ inline float softplus(float x)
{
    const float e = exp_fast(x), u = 1.f + e;
    const float r = __builtin_amdgcn_logf(u) * 0.69314718055994530942f + (u < 4.f ? e - (u - 1.f) : 0.f);
    return x > 20.f ? x : r;
}

// A sum of any number of values: off by one rounding of it, and by n * 2^-47 of the n values' magnitudes.  What an addition loses is a number of 32 bits again and
// is summed by itself (Knuth, The Art of Computer Programming, 4.2.2, theorem B).  A sum past the range stays infinite.
struct LongSum {
    float s = 0.f, lost = 0.f;
    __device__ void add(float v)
    {
        const float t = s + v, of_v = t - s;
        lost += (s - (t - of_v)) + (v - of_v);
        s = t;
    }
    __device__ float total() const { return lost == lost ? s + lost : s; }
};

// a number as a type, for what chooses a kernel's template arguments
template <int V> struct SeqInt { static constexpr int value = V; };

inline int div_up(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// a slot index of a step call: row -> slot, or -1 for a row to skip
__device__ inline int step_slot(const int32_t *slots, int row, int num_slots)
{
    const int s = slots ? slots[row] : row;
    return s >= 0 && s < num_slots ? s : -1;
}

// ---- launchers (seq_conv1d.hip, seq_headnorm.hip, seq_scan.hip, seq_scan_bwd.hip); arguments checked by seq_api.hip ----
hipError_t launch_conv1d_fwd(const void *x, const void *w, const float *bias, void *y, const sn_conv1d_shape &s, const int32_t *off,
                             const void *state_in, void *state_out, hipStream_t st);
size_t conv1d_scratch_bytes(int64_t rows, int channels, int width);
hipError_t launch_conv1d_bwd(const void *x, const void *w, const float *bias, const void *dy, void *dx, float *dw, float *dbias,
                             const sn_conv1d_shape &s, const int32_t *off, const void *state_in, const void *dstate_out,
                             void *dstate_in, void *scratch, hipStream_t st);
hipError_t launch_conv1d_step(const void *x, const void *w, const float *bias, void *y, const void *state, void *state_out,
                              const int32_t *slots, int num_slots, const sn_conv1d_shape &s, hipStream_t st);
hipError_t launch_headnorm_fwd(const void *q, const void *k, const float *wq, const float *wk, const int32_t *pos, const float *freq,
                               void *yq, void *yk, const sn_headnorm_shape &s, hipStream_t st);
size_t headnorm_scratch_bytes(int64_t rows, int q_heads, int k_heads, int head_dim);
hipError_t launch_headnorm_bwd(const void *q, const void *k, const float *wq, const float *wk, const int32_t *pos, const float *freq,
                               const void *dyq, const void *dyk, void *dq, void *dk, float *dwq, float *dwk,
                               const sn_headnorm_shape &s, void *scratch, hipStream_t st);
void scan_bwd_bytes(const sn_scan_shape &s, size_t *min_bytes, size_t *preferred_bytes);   // without the states
void scan_fwd_bytes(const sn_scan_shape &s, size_t *preferred_bytes);
size_t scan_states_bytes(const sn_scan_shape &s);
hipError_t launch_scan_fwd(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z, const float *bias, void *y,
                           const sn_scan_shape &s, const int32_t *off, const float *h0, float *hT, float *states, void *ws, size_t ws_bytes, hipStream_t st);
struct ScanGrads {
    const void *dy;
    void *du, *ddt, *dB, *dC, *dz;
    float *dA, *dD, *ddt_bias, *dh0;
    const float *dhT;
};
hipError_t launch_scan_bwd(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z, const float *bias,
                           const ScanGrads &g, const sn_scan_shape &s, const int32_t *off, const float *h0, const float *states, void *ws, size_t ws_bytes, hipStream_t st);
hipError_t launch_scan_step(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z, const float *bias, void *y,
                            const float *state, float *state_out, const int32_t *slots, int num_slots, const sn_scan_shape &s, hipStream_t st);

}  // namespace sn
