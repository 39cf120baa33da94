// How the kernels of the token-sequence layers walk along the rows of packed sequences.  Whole numbers only: with an empty __device__ it is host code as well,
// and is tested as such with offsets of all kinds.
#pragma once
#include <cstdint>

namespace sn {

// The rows of packed sequences: off == nullptr: `seqs` sequences of `len` rows.  A row of no sequence has s outside 0 .. seqs - 1.  begin
// and end stay within 0 .. rows whatever the offsets hold.
struct SeqRows {
    const int32_t *off;
    int seqs, len, rows;
};
struct SeqAt {
    int s, begin, end;  // the sequence of a row, its first row and the one behind its last
    __device__ bool holds(int row, const SeqRows &r) const { return s >= 0 && s < r.seqs && begin <= row && row < end; }
};
__device__ inline SeqAt seq_clamped(const SeqRows &r, int s)
{
    SeqAt a;
    a.s = s;
    a.begin = s < 0 ? 0 : min(max(r.off[s], 0), r.rows);
    a.end = s < r.seqs ? min(max(r.off[s + 1], 0), r.rows) : r.rows;
    return a;
}
// The last sequence that begins at or before `row` (s = -1: none does; s = seqs: the row lies behind all of them).
__device__ inline SeqAt seq_find(const SeqRows &r, int row)
{
    if (!r.off) {
        SeqAt a;
        a.s = row / r.len;
        a.begin = a.s * r.len;
        a.end = a.begin + r.len;
        return a;
    }
    int lo = -1, hi = r.seqs + 1;  // off[lo] <= row < off[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (r.off[mid] <= row) lo = mid; else hi = mid;
    }
    return seq_clamped(r, lo);
}
// From the place of an earlier row on to that of `row`.  The next sequence mostly holds it; empty ones are passed by jumps that double as long as they do not go too
// far, and else become half as long.
__device__ inline void seq_forward(const SeqRows &r, SeqAt &a, int row)
{
    for (int jump = 0; a.s < r.seqs && row >= a.end;) {
        if (r.off) {
            int s = a.s + 1;   // off[s] <= row
            if (jump) {
                const bool near = jump <= r.seqs - s && r.off[s + jump] <= row;
                s = near ? s + jump : s;
                jump = near ? 2 * jump : (jump + 1) / 2;
            } else {
                jump = 1;
            }
            a = seq_clamped(r, s);
        } else {
            ++a.s;
            a.begin = a.end;
            a.end = a.s < r.seqs ? a.end + r.len : r.rows;   // behind the last, the sum could pass 32 bits
        }
    }
}

// The rows p0 .. p1 - 1 that one turn of a kernel's loop works on: those of one sequence in the tile of rows t0 .. t0 + ROWS - 1.  The tile's other
// rows are staged as zeros: delta = 0 leaves the states, and the gradient on its way through them, as they are.
struct Piece {
    int t0, p0, p1, seq;
    bool any, start, end;   // whether there is one; it begins, ends its sequence
    __device__ bool holds(int row) const { return any && row >= p0 && row < p1; }
};
// The first piece at or behind row `from` of the chunk r0 .. r1 - 1.  `at`: the place of an earlier row.
template <int ROWS> __device__ inline Piece piece_from(const SeqRows &r, SeqAt &at, int from, int r0, int r1)
{
    Piece p = {};
    if (at.s < 0 && from < r1) at = seq_clamped(r, 0);
    from = max(from, at.begin);
    seq_forward(r, at, from);
    from = max(from, at.begin);
    if (at.s >= r.seqs || from >= r1 || from >= at.end) return p;
    p.any = true;
    p.seq = at.s;
    p.p0 = from;
    p.t0 = r0 + (from - r0) / ROWS * ROWS;
    p.p1 = min(min(p.t0 + ROWS, at.end), r1);
    p.start = from == at.begin;
    p.end = p.p1 == at.end;
    return p;
}
// The last piece in front of row `to`.  `at`: the place of a later row.
template <int ROWS> __device__ inline Piece piece_before(const SeqRows &r, SeqAt &at, int to, int r0)
{
    Piece p = {};
    if (at.s >= r.seqs && to > r0) at = seq_clamped(r, r.seqs - 1);
    to = min(to, at.end);
    for (int turn = 0; turn < 2 && at.s >= 0 && to > r0 && to <= at.begin; ++turn) {   // the one in front, or, where that is empty, the last one that is not
        if (at.s == 0) at = SeqAt{-1, 0, 0};
        else if (turn) at = seq_find(r, to - 1);
        else at = r.off ? seq_clamped(r, at.s - 1) : SeqAt{at.s - 1, at.begin - r.len, at.begin};
        to = min(to, at.end);
    }
    if (at.s < 0 || at.s >= r.seqs || to <= r0 || to <= at.begin) return p;
    p.any = true;
    p.seq = at.s;
    p.p1 = to;
    p.t0 = r0 + (to - 1 - r0) / ROWS * ROWS;
    p.p0 = max(p.t0, at.begin);
    p.start = p.p0 == at.begin;
    p.end = to == at.end;
    return p;
}

}  // namespace sn
