// The walk of the token-sequence kernels along packed rows (csrc/seq_walk.h) as host code, for the AddressSanitizer / UBSan build of the CPU test suite: every
// loop of the kernels that moves from piece to piece or row to row, with offsets of all kinds.  Offsets that descend or leave the rows
// may give any result, but no row outside of the tensors, no sequence that there is not, and no loop without an end; valid ones give each row that a
// sequence holds once, in its sequence.  Exit status 0 = all of it held and the sanitizers found nothing.
#include <algorithm>
#include <chrono>
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#define __device__
using std::max;
using std::min;
#include "seq_walk.h"

#define CHECK(c) do { if (!(c)) { std::fprintf(stderr, "walk driver: check failed at line %d: %s\n", __LINE__, #c); std::exit(2); } } while (0)
using namespace sn;

namespace {
std::mt19937 rng(7);
int upto(int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); }

struct Case {
    SeqRows r;
    bool valid;
    std::vector<int> owner;                      // valid: the sequence of each row, -1: none
    int begin(int s) const { return r.off ? r.off[s] : s * r.len; }
    int end(int s) const { return begin(s + 1); }
};

void check_piece(const Case &c, const Piece &p, int rows, int r0, int r1)
{
    CHECK(p.any && p.seq >= 0 && p.seq < c.r.seqs);
    CHECK(r0 <= p.t0 && p.t0 <= p.p0 && p.p0 < p.p1 && p.p1 <= p.t0 + rows && p.p1 <= r1 && r1 <= c.r.rows && (p.t0 - r0) % rows == 0);
    if (!c.valid) return;
    for (int t = p.p0; t < p.p1; ++t) CHECK(c.owner[t] == p.seq);
    CHECK(p.start == (p.p0 == c.begin(p.seq)) && p.end == (p.p1 == c.end(p.seq)));
}

// Forward through a chunk, from row `from` on: the rows seen, and how often.
template <int ROWS> void forward(const Case &c, int r0, int r1, bool last_only, std::vector<int> &seen)
{
    SeqAt at = seq_find(c.r, last_only ? r1 - 1 : r0);
    const int from = last_only ? max(r0, at.begin) : r0;
    Piece p = piece_from<ROWS>(c.r, at, from, r0, r1);
    for (int turns = 0; p.any; ++turns) {
        CHECK(turns <= r1 - r0);
        check_piece(c, p, ROWS, r0, r1);
        for (int t = p.p0; t < p.p1; ++t) ++seen[t];
        const Piece q = piece_from<ROWS>(c.r, at, p.p1, r0, r1);
        if (q.any) CHECK(q.p0 >= p.p1);
        p = q;
    }
    if (c.valid && last_only)   // all of the chunk's rows of the sequence that holds its last row
        for (int t = r0; t < r1; ++t) CHECK(seen[t] == (c.owner[r1 - 1] >= 0 && c.owner[t] == c.owner[r1 - 1]));
}

void backward(const Case &c, int r0, int r1, bool first_only, std::vector<int> &seen)
{
    SeqAt at = seq_find(c.r, first_only ? r0 : r1 - 1);
    Piece p = piece_before<16>(c.r, at, first_only ? min(r1, at.end) : r1, r0);
    for (int turns = 0; p.any; ++turns) {
        CHECK(turns <= r1 - r0);
        check_piece(c, p, 16, r0, r1);
        for (int t = p.p0; t < p.p1; ++t) ++seen[t];
        const Piece q = piece_before<16>(c.r, at, p.p0, r0);
        if (q.any) CHECK(q.p1 <= p.p0);
        p = q;
    }
    if (c.valid && first_only)
        for (int t = r0; t < r1; ++t) CHECK(seen[t] == (c.owner[r0] >= 0 && c.owner[t] == c.owner[r0]));
}

// The convolution: row by row from a place on.
void rows_of(const Case &c, int r0, int r1, int back)
{
    SeqAt at = seq_find(c.r, max(r0 - back, 0));
    for (int t = r0 - back; t < r1; ++t) {
        seq_forward(c.r, at, t);
        const bool there = t >= 0 && at.holds(t, c.r);
        if (there) CHECK(at.s >= 0 && at.s < c.r.seqs && at.begin >= 0 && at.begin <= t && t < at.end && at.end <= c.r.rows);
        if (c.valid && t >= 0) CHECK(there == (c.owner[t] >= 0) && (!there || at.s == c.owner[t]));
    }
}

void walk(const Case &c)
{
    const int rows = c.r.rows;
    if (c.r.off)
        for (int s = 0; s < c.r.seqs; ++s) {
            const SeqAt at = seq_clamped(c.r, s);
            CHECK(0 <= at.begin && at.begin <= rows && 0 <= at.end && at.end <= rows);
        }
    for (const int chunk : {16, 32, 48, 16 * ((rows + 15) / 16)}) {
        std::vector<int> f32(rows), f16(rows), b(rows);
        for (int r0 = 0; r0 < rows; r0 += chunk) {
            const int r1 = min(r0 + chunk, rows);
            forward<32>(c, r0, r1, false, f32);
            forward<16>(c, r0, r1, false, f16);
            backward(c, r0, r1, false, b);
            std::vector<int> last(rows), first(rows);
            forward<32>(c, r0, r1, true, last);
            backward(c, r0, r1, true, first);
            rows_of(c, r0, r1, 0);
            rows_of(c, r0, r1, 5);
        }
        if (c.valid)
            for (int t = 0; t < rows; ++t) CHECK(f32[t] == (c.owner[t] >= 0) && f16[t] == f32[t] && b[t] == f32[t]);
    }
}
}  // namespace

int main()
{
    for (int i = 0; i < 60000; ++i) {
        const int seqs = upto(1, i % 3 ? 6 : 40), kind = i % 6, rows = upto(1, 140);
        std::vector<int32_t> off(seqs + 1);   // its bounds are the sanitizer's to watch
        Case c = {{off.data(), seqs, 0, rows}, kind < 3, {}};
        for (auto &o : off) o = kind == 3 ? upto(-20, rows + 20) : upto(0, rows);
        if (kind < 3) std::sort(off.begin(), off.end());
        if (kind == 1) off.front() = 0, off.back() = rows;
        if (kind == 4) std::sort(off.rbegin(), off.rend());
        if (kind == 5)
            for (auto &o : off) {
                const int32_t ends[] = {INT_MIN, INT_MAX, -1, 0, rows, rows + 1, upto(0, rows)};
                o = ends[upto(0, 6)];
            }
        if (c.valid) {
            c.owner.assign(rows, -1);
            for (int s = 0; s < seqs; ++s)
                for (int t = off[s]; t < off[s + 1]; ++t) c.owner[t] = s;
        }
        walk(c);
    }
    for (int i = 0; i < 5000; ++i) {   // equal lengths
        const int seqs = upto(1, 30), len = upto(1, 50);
        Case c = {{nullptr, seqs, len, seqs * len}, true, {}};
        for (int t = 0; t < seqs * len; ++t) c.owner.push_back(t / len);
        walk(c);
    }
    // empty sequences, the most that a call may have, between two of eight rows: passed in a few steps (one after the other takes minutes here)
    {
        const int seqs = (1 << 24) - 1;
        std::vector<int32_t> off(seqs + 1, 8);
        off.front() = 0;
        off.back() = 16;
        const SeqRows r = {off.data(), seqs, 0, 16};
        const auto start = std::chrono::steady_clock::now();
        for (int i = 0; i < 1000; ++i) {
            SeqAt at = seq_find(r, 0);
            Piece p = piece_from<16>(r, at, 0, 0, 16);
            CHECK(p.any && p.seq == 0 && p.p1 == 8);
            p = piece_from<16>(r, at, 8, 0, 16);
            CHECK(p.any && p.seq == seqs - 1 && p.p0 == 8 && p.p1 == 16 && p.start && p.end);
            p = piece_before<16>(r, at, 8, 0);
            CHECK(p.any && p.seq == 0 && p.p0 == 0 && p.p1 == 8 && p.start && p.end);
            at = seq_find(r, 3);
            seq_forward(r, at, 8);
            CHECK(at.s == seqs - 1 && at.begin == 8 && at.end == 16);
        }
        CHECK(std::chrono::duration<double>(std::chrono::steady_clock::now() - start).count() < 5);
    }
    // the most rows that a call may have, in one sequence: nothing passes 32 bits at its end
    const int most = 1 << 30;
    for (const int seqs : {1, 2}) {
        const SeqRows r = {nullptr, seqs, most / seqs, most};
        SeqAt at = seq_find(r, most - 1);
        CHECK(at.s == seqs - 1 && at.end == most);
        Piece p = piece_from<32>(r, at, most - 40, most - 64, most);
        while (p.any) p = piece_from<32>(r, at, p.p1, most - 64, most);
        at = seq_find(r, most - 1);
        seq_forward(r, at, most + 16);
        CHECK(!at.holds(most, r));
        at = seq_find(r, most - 1);
        p = piece_before<16>(r, at, most, 0);
        CHECK(p.any && p.end && p.p1 == most);
    }
    std::puts("walk driver: ok");
    return 0;
}
