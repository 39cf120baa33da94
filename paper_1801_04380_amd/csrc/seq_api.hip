// Host side of sn_seq.h: what a call is given is checked here, before anything is launched.
#include "seq.h"

using namespace sn;

namespace {

constexpr int64_t INT32_MOST = 0x7fffffffLL;
constexpr int64_t ROWS_MOST = 1 << 30;            // the kernels look a tile further in 32 bits
constexpr int64_t GRID_MOST = (1 << 24) - 1;      // workgroups of 256 threads in a grid's first dimension: sequences, rows of a step
constexpr int64_t GRID_Y_MOST = 65535;            // and in its second: blocks of channels

bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
size_t esize(int dtype) { return dtype == SN_BF16 ? 2 : 4; }
bool flag(int v) { return v == 0 || v == 1; }
bool valid_dtype(int d) { return d == SN_F32 || d == SN_BF16; }

sn_status launched(hipError_t e) { return e == hipSuccess ? SN_OK : SN_ERR_LAUNCH; }

// A tensor that has to be there unless it has no rows, and one that may be absent.
bool tensor(const void *p, size_t align, int64_t rows) { return rows == 0 || (p && aligned(p, align)); }
bool optional(const void *p, size_t align) { return aligned(p, align); }

// Rows of `width` elements that are ld apart; of a single row the stride does not matter.
bool stride(int64_t ld, int64_t width, int64_t rows) { return rows <= 1 || (ld >= width && ld <= INT32_MOST); }

bool same(const void *a, const void *b) { return a && a == b; }

// Two dense fp32 arrays of n elements that share some.
bool overlap(const float *a, const float *b, size_t n) { return a && b && a < b + n && b < a + n; }

sn_status check_rows(int64_t rows, int32_t seqs, bool ragged)
{
    if (rows < 0 || seqs < 1) return SN_ERR_BAD_ARG;
    if (!ragged && rows % seqs) return SN_ERR_BAD_ARG;
    if (rows > ROWS_MOST || seqs > GRID_MOST) return SN_ERR_UNSUPPORTED;
    return SN_OK;
}

sn_status check_conv1d(const sn_conv1d_shape *s, const void *x, const void *w, const float *bias, const void *y)
{
    if (!s || s->rows < 0 || s->channels < 1 || s->width < 1 || !valid_dtype(s->dtype) || !flag(s->silu)) return SN_ERR_BAD_ARG;
    if (s->width > SN_CONV1D_MAX_WIDTH || s->rows > ROWS_MOST) return SN_ERR_UNSUPPORTED;
    const size_t e = esize(s->dtype);
    if (!tensor(x, e, s->rows) || !tensor(y, e, s->rows) || !w || !aligned(w, e) || !optional(bias, 4) || same(x, y)) return SN_ERR_BAD_ARG;
    if (!stride(s->ld_x, s->channels, s->rows) || !stride(s->ld_y, s->channels, s->rows)) return SN_ERR_BAD_ARG;
    if (s->channels > GRID_Y_MOST * 256) return SN_ERR_UNSUPPORTED;
    return SN_OK;
}

// The states of a step call; width - 1 may be 0, and then there is none.
sn_status check_slots(const void *state, const void *state_out, size_t align, const int32_t *slots, int32_t num_slots, int64_t rows, bool none)
{
    if (num_slots < 0 || (!none && rows && num_slots && (!state || !state_out)) || !aligned(state, align) || !aligned(state_out, align) || !aligned(slots, 4))
        return SN_ERR_BAD_ARG;
    if (!slots && rows > num_slots) return SN_ERR_BAD_ARG;
    return rows > GRID_MOST ? SN_ERR_UNSUPPORTED : SN_OK;
}

sn_status check_headnorm(const sn_headnorm_shape *s, const void *q, const void *k, const float *wq, const float *wk, const int32_t *positions, const float *inv_freq,
                         const void *yq, const void *yk)
{
    if (!s || s->rows < 0 || s->q_heads < 1 || s->k_heads < 0 || s->head_dim < 2 || s->head_dim % 2 || s->rot_dim < 0 || s->rot_dim % 2 || s->rot_dim > s->head_dim ||
        !flag(s->interleaved) || !valid_dtype(s->dtype) || !(s->eps > 0.f))
        return SN_ERR_BAD_ARG;
    if (s->head_dim > SN_HEADNORM_MAX_DIM || s->rows > ROWS_MOST || (int64_t)s->q_heads + s->k_heads > (1 << 20)) return SN_ERR_UNSUPPORTED;
    const size_t e = esize(s->dtype);
    const int64_t nq = (int64_t)s->q_heads * s->head_dim, nk = (int64_t)s->k_heads * s->head_dim;
    if (!tensor(q, e, s->rows) || !tensor(yq, e, s->rows) || !stride(s->ld_q, nq, s->rows) || !stride(s->ld_yq, nq, s->rows)) return SN_ERR_BAD_ARG;
    if (s->k_heads && (!tensor(k, e, s->rows) || !tensor(yk, e, s->rows) || !stride(s->ld_k, nk, s->rows) || !stride(s->ld_yk, nk, s->rows))) return SN_ERR_BAD_ARG;
    if (!optional(wq, 4) || !optional(wk, 4) || !optional(positions, 4) || !optional(inv_freq, 4) || (s->rot_dim && !inv_freq)) return SN_ERR_BAD_ARG;
    return SN_OK;
}

// What of a scan's shape does not depend on strides; rows and seqs as check_rows.
sn_status check_scan_sizes(const sn_scan_shape *s)
{
    if (!s || s->channels < 1 || s->states < 1 || s->groups < 1 || s->channels % s->groups || !valid_dtype(s->dtype) || !flag(s->softplus) || !flag(s->ragged))
        return SN_ERR_BAD_ARG;
    if (s->states > SN_SCAN_MAX_STATES || s->groups * (int64_t)((s->channels / s->groups + 15) / 16) > GRID_Y_MOST) return SN_ERR_UNSUPPORTED;
    return check_rows(s->rows, s->seqs, s->ragged);
}

// The kernels keep a row's stride in 32 bits, the place in a tile of 32 rows in as many.
bool wide(int64_t ld) { return ld > (1 << 24); }

sn_status check_scan(const sn_scan_shape *s, const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z, const float *bias,
                     const void *y)
{
    const sn_status st = check_scan_sizes(s);
    if (st != SN_OK) return st;
    const size_t e = esize(s->dtype);
    const int64_t gn = (int64_t)s->groups * s->states;
    if (!tensor(u, e, s->rows) || !tensor(dt, e, s->rows) || !tensor(B, e, s->rows) || !tensor(C, e, s->rows) || !tensor(y, e, s->rows) || !A || !aligned(A, 4) ||
        !optional(D, 4) || !optional(z, e) || !optional(bias, 4))
        return SN_ERR_BAD_ARG;
    if (!stride(s->ld_u, s->channels, s->rows) || !stride(s->ld_dt, s->channels, s->rows) || !stride(s->ld_b, gn, s->rows) || !stride(s->ld_c, gn, s->rows) ||
        !stride(s->ld_y, s->channels, s->rows) || (z && !stride(s->ld_z, s->channels, s->rows)))
        return SN_ERR_BAD_ARG;
    if (s->rows > 1 && (wide(s->ld_u) || wide(s->ld_dt) || wide(s->ld_b) || wide(s->ld_c) || wide(s->ld_y) || (z && wide(s->ld_z)))) return SN_ERR_UNSUPPORTED;
    return SN_OK;
}

}  // namespace

extern "C" {

sn_status sn_causal_conv1d_fwd(const void *x, const void *w, const float *bias, void *y, const sn_conv1d_shape *shape, const int32_t *seq_offsets,
                               const void *state_in, void *state_out, sn_stream stream)
{
    sn_status s = check_conv1d(shape, x, w, bias, y);
    if (s != SN_OK) return s;
    s = check_rows(shape->rows, shape->seqs, seq_offsets != nullptr);
    if (s != SN_OK) return s;
    const size_t e = esize(shape->dtype);
    if (!aligned(seq_offsets, 4) || !optional(state_in, e) || !optional(state_out, e) || same(state_in, state_out)) return SN_ERR_BAD_ARG;
    if (shape->rows == 0 && !state_out) return SN_OK;
    return launched(launch_conv1d_fwd(x, w, bias, y, *shape, seq_offsets, state_in, state_out, static_cast<hipStream_t>(stream)));
}

size_t sn_causal_conv1d_scratch_bytes(int64_t rows, int32_t channels, int32_t width)
{
    if (rows < 0 || rows > ROWS_MOST || channels < 1 || width < 1 || width > SN_CONV1D_MAX_WIDTH || channels > GRID_Y_MOST * 256) return 0;
    return conv1d_scratch_bytes(rows, channels, width);
}

sn_status sn_causal_conv1d_bwd(const void *x, const void *w, const float *bias, const void *dy, void *dx, float *dw, float *dbias, const sn_conv1d_shape *shape,
                               const int32_t *seq_offsets, const void *state_in, const void *dstate_out, void *dstate_in, void *scratch, size_t scratch_bytes,
                               sn_stream stream)
{
    sn_status s = check_conv1d(shape, x, w, bias, dy);
    if (s != SN_OK) return s;
    s = check_rows(shape->rows, shape->seqs, seq_offsets != nullptr);
    if (s != SN_OK) return s;
    const size_t e = esize(shape->dtype);
    if (!tensor(dx, e, shape->rows) || !stride(shape->ld_dx, shape->channels, shape->rows) || same(x, dx) || same(dy, dx) || !dw || !aligned(dw, 4) ||
        !optional(dbias, 4) || !aligned(seq_offsets, 4) || !optional(state_in, e) || !optional(dstate_out, e) || !optional(dstate_in, e) ||
        same(dstate_in, dstate_out) || same(dstate_in, state_in) || !scratch || !aligned(scratch, 256))
        return SN_ERR_BAD_ARG;
    if (scratch_bytes < conv1d_scratch_bytes(shape->rows, shape->channels, shape->width)) return SN_ERR_WORKSPACE_TOO_SMALL;
    return launched(launch_conv1d_bwd(x, w, bias, dy, dx, dw, dbias, *shape, seq_offsets, state_in, dstate_out, dstate_in, scratch, static_cast<hipStream_t>(stream)));
}

sn_status sn_causal_conv1d_step(const void *x, const void *w, const float *bias, void *y, const void *state, void *state_out, const int32_t *slots, int32_t num_slots,
                                const sn_conv1d_shape *shape, sn_stream stream)
{
    sn_status s = check_conv1d(shape, x, w, bias, y);
    if (s != SN_OK) return s;
    s = check_slots(state, state_out, esize(shape->dtype), slots, num_slots, shape->rows, shape->width == 1);
    if (s != SN_OK || shape->rows == 0) return s;
    return launched(launch_conv1d_step(x, w, bias, y, state, state_out, slots, num_slots, *shape, static_cast<hipStream_t>(stream)));
}

sn_status sn_headnorm_rot_fwd(const void *q, const void *k, const float *wq, const float *wk, const int32_t *positions, const float *inv_freq, void *yq, void *yk,
                              const sn_headnorm_shape *shape, sn_stream stream)
{
    const sn_status s = check_headnorm(shape, q, k, wq, wk, positions, inv_freq, yq, yk);
    if (s != SN_OK || shape->rows == 0) return s;
    if ((same(q, yq) && shape->ld_q != shape->ld_yq) || (shape->k_heads && same(k, yk) && shape->ld_k != shape->ld_yk)) return SN_ERR_BAD_ARG;
    return launched(launch_headnorm_fwd(q, k, wq, wk, positions, inv_freq, yq, yk, *shape, static_cast<hipStream_t>(stream)));
}

size_t sn_headnorm_rot_scratch_bytes(int64_t rows, int32_t q_heads, int32_t k_heads, int32_t head_dim)
{
    if (rows < 0 || rows > ROWS_MOST || q_heads < 1 || k_heads < 0 || (int64_t)q_heads + k_heads > (1 << 20) || head_dim < 2 || head_dim > SN_HEADNORM_MAX_DIM) return 0;
    return headnorm_scratch_bytes(rows, q_heads, k_heads, head_dim);
}

sn_status sn_headnorm_rot_bwd(const void *q, const void *k, const float *wq, const float *wk, const int32_t *positions, const float *inv_freq, const void *dyq,
                              const void *dyk, void *dq, void *dk, float *dwq, float *dwk, const sn_headnorm_shape *shape, void *scratch, size_t scratch_bytes,
                              sn_stream stream)
{
    const sn_status s = check_headnorm(shape, q, k, wq, wk, positions, inv_freq, dyq, dyk);
    if (s != SN_OK) return s;
    const size_t e = esize(shape->dtype);
    const int64_t nq = (int64_t)shape->q_heads * shape->head_dim, nk = (int64_t)shape->k_heads * shape->head_dim;
    if (!tensor(dq, e, shape->rows) || !stride(shape->ld_dq, nq, shape->rows) || same(q, dq) || (same(dyq, dq) && shape->ld_yq != shape->ld_dq)) return SN_ERR_BAD_ARG;
    if (shape->k_heads && (!tensor(dk, e, shape->rows) || !stride(shape->ld_dk, nk, shape->rows) || same(k, dk) || (same(dyk, dk) && shape->ld_yk != shape->ld_dk)))
        return SN_ERR_BAD_ARG;
    if (!optional(dwq, 4) || !optional(dwk, 4) || !scratch || !aligned(scratch, 256)) return SN_ERR_BAD_ARG;
    if (scratch_bytes < headnorm_scratch_bytes(shape->rows, shape->q_heads, shape->k_heads, shape->head_dim)) return SN_ERR_WORKSPACE_TOO_SMALL;
    return launched(launch_headnorm_bwd(q, k, wq, wk, positions, inv_freq, dyq, dyk, dq, dk, dwq, dwk, *shape, scratch, static_cast<hipStream_t>(stream)));
}

sn_status sn_scan_workspace_query(const sn_scan_shape *shape, sn_scan_dir dir, size_t *min_bytes, size_t *preferred_bytes)
{
    const sn_status s = check_scan_sizes(shape);
    if (s != SN_OK) return s;
    if (!min_bytes || !preferred_bytes || (dir != SN_SCAN_FWD && dir != SN_SCAN_BWD)) return SN_ERR_BAD_ARG;
    if (dir == SN_SCAN_FWD) {
        *min_bytes = 0;
        scan_fwd_bytes(*shape, preferred_bytes);
    } else {
        scan_bwd_bytes(*shape, min_bytes, preferred_bytes);
    }
    return SN_OK;
}

size_t sn_scan_states_bytes(const sn_scan_shape *shape) { return check_scan_sizes(shape) == SN_OK ? scan_states_bytes(*shape) : 0; }

sn_status sn_scan_fwd(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z, const float *dt_bias, void *y,
                      const sn_scan_shape *shape, const int32_t *seq_offsets, const float *h0, float *hT, float *states, void *workspace, size_t workspace_bytes,
                      sn_stream stream)
{
    const sn_status s = check_scan(shape, u, dt, A, B, C, D, z, dt_bias, y);
    if (s != SN_OK) return s;
    if ((seq_offsets != nullptr) != (shape->ragged != 0) || !aligned(seq_offsets, 4) || !optional(h0, 4) || !optional(hT, 4) || !optional(states, 256) || same(u, y) ||
        same(dt, y) || same(z, y) || overlap(h0, hT, (size_t)shape->seqs * shape->channels * shape->states) || (workspace_bytes && !workspace) ||
        !aligned(workspace, 256))
        return SN_ERR_BAD_ARG;
    if (shape->rows == 0 && !hT) return SN_OK;
    return launched(launch_scan_fwd(u, dt, A, B, C, D, z, dt_bias, y, *shape, seq_offsets, h0, hT, states, workspace, workspace_bytes, static_cast<hipStream_t>(stream)));
}

sn_status sn_scan_bwd(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z, const float *dt_bias, const void *dy,
                      void *du, void *ddt, float *dA, void *dB, void *dC, float *dD, void *dz, float *ddt_bias, const sn_scan_shape *shape, const int32_t *seq_offsets,
                      const float *h0, const float *states, const float *dhT, float *dh0, void *workspace, size_t workspace_bytes, sn_stream stream)
{
    const sn_status s = check_scan(shape, u, dt, A, B, C, D, z, dt_bias, dy);
    if (s != SN_OK) return s;
    const size_t e = esize(shape->dtype);
    const int64_t rows = shape->rows, gn = (int64_t)shape->groups * shape->states;
    if ((seq_offsets != nullptr) != (shape->ragged != 0) || !aligned(seq_offsets, 4) || !optional(h0, 4) || !optional(states, 256) || !optional(dhT, 4) || !optional(dh0, 4) ||
        overlap(dhT, dh0, (size_t)shape->seqs * shape->channels * shape->states) || overlap(h0, dh0, (size_t)shape->seqs * shape->channels * shape->states))
        return SN_ERR_BAD_ARG;
    if (!tensor(du, e, rows) || !tensor(ddt, e, rows) || !tensor(dB, e, rows) || !tensor(dC, e, rows) || !dA || !aligned(dA, 4) || (dD != nullptr) != (D != nullptr) ||
        !aligned(dD, 4) || (ddt_bias != nullptr) != (dt_bias != nullptr) || !aligned(ddt_bias, 4) || (rows && (dz != nullptr) != (z != nullptr)) || !optional(dz, e))
        return SN_ERR_BAD_ARG;
    if (!stride(shape->ld_du, shape->channels, rows) || !stride(shape->ld_ddt, shape->channels, rows) || !stride(shape->ld_db, gn, rows) || !stride(shape->ld_dc, gn, rows) ||
        (dz && !stride(shape->ld_dz, shape->channels, rows)))
        return SN_ERR_BAD_ARG;
    if (rows > 1 && (wide(shape->ld_du) || wide(shape->ld_ddt) || wide(shape->ld_db) || wide(shape->ld_dc) || (dz && wide(shape->ld_dz)))) return SN_ERR_UNSUPPORTED;
    const void *in[] = {u, dt, z, dy, B, C}, *out[] = {du, ddt, dz, dB, dC};
    for (const void *o : out) {
        for (const void *i : in)
            if (same(o, i)) return SN_ERR_BAD_ARG;
        int times = 0;
        for (const void *p : out) times += same(o, p);
        if (times > 1) return SN_ERR_BAD_ARG;
    }
    if (!workspace || !aligned(workspace, 256)) return SN_ERR_BAD_ARG;
    size_t least, preferred;
    scan_bwd_bytes(*shape, &least, &preferred);
    if (workspace_bytes < least + (states ? 0 : scan_states_bytes(*shape))) return SN_ERR_WORKSPACE_TOO_SMALL;
    const ScanGrads g = {dy, du, ddt, dB, dC, dz, dA, dD, ddt_bias, dh0, dhT};
    return launched(launch_scan_bwd(u, dt, A, B, C, D, z, dt_bias, g, *shape, seq_offsets, h0, states, workspace, workspace_bytes, static_cast<hipStream_t>(stream)));
}

sn_status sn_scan_step(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z, const float *dt_bias, void *y,
                       const float *state, float *state_out, const int32_t *slots, int32_t num_slots, const sn_scan_shape *shape, sn_stream stream)
{
    if (!shape) return SN_ERR_BAD_ARG;
    sn_scan_shape one = *shape;   // its rows are streams, not a sequence
    one.seqs = 1;
    one.ragged = 0;
    sn_status s = check_scan(&one, u, dt, A, B, C, D, z, dt_bias, y);
    if (s != SN_OK) return s;
    if (same(u, y) || same(dt, y) || same(z, y)) return SN_ERR_BAD_ARG;
    s = check_slots(state, state_out, 4, slots, num_slots, one.rows, false);
    if (s != SN_OK || one.rows == 0) return s;
    return launched(launch_scan_step(u, dt, A, B, C, D, z, dt_bias, y, state, state_out, slots, num_slots, one, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
