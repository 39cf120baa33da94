"""The scan over many sequences of equal length that share tiles and chunks although each is longer than a tile."""
import pytest
import torch

import paper_1801_04380_amd as sn
from test_gpu_seq import Scan, Out, bytes_, close, offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,S,L,N", [("bf16", 8200, 17, 16), ("f32", 8193, 33, 5), ("f32", 8193, 17, 20)])
def test_scan_of_many_sequences_of_a_few_tiles(dtype, S, L, N):
    """As ragged sequences and as equal ones the rows are cut in the same way, and the results are the same, with any workspace; the first
    sequences and the last ones against the oracle."""
    c = Scan(dtype, [L] * S, S * L, 24, N, 1, S + L)
    some, last = 5, S - 3
    pick = slice(0, some * L), slice(last * L, S * L)
    parts = []
    for at, first, n in ((pick[0], 0, some), (pick[1], last, S - last)):
        p = Scan(dtype, [L] * n, n * L, 24, N, 1, 0)
        p.f = [t if k in ("A", "D", "bias") or t is None else t[at] for k, t in zip(c.t, c.f)]
        p.dy, p.h0, p.dhT = c.dy[at], c.h0[first:first + n], c.dhT[first:first + n]
        parts.append((at, slice(first, first + n), p.want()))
    for full in (False, True):
        kept = []
        for off in (None, offsets([L] * S)):
            kw, shape = {"seqs": S, "offsets": off}, c.shape(off is not None)
            fwd, bwd = (sn.sn_scan_workspace_query(shape, i)[int(full)] for i in (sn.SN_SCAN_FWD, sn.SN_SCAN_BWD))
            states = bytes_(sn.sn_scan_states_bytes(shape))
            gy, gh = c.forward(kw, states, bytes_(fwd))
            g = c.backward(kw, bytes_(bwd), states)
            kept.append([gy.wide, gh] + [v.wide if isinstance(v, Out) else v for v in g.values() if v is not None])
            for at, seq, (y, hT, want) in parts:
                close(gy.t[at], y, c.d.dtype)
                close(gh[seq], hT)
                close(g["dh0"][seq], want["dh0"])
                for k in ("du", "ddt", "dB", "dC", "dz"):
                    close(g[k].t[at], want[k], c.d.dtype)
        assert all(torch.equal(a, b) for a, b in zip(*kept))
        # a call that keeps no states walks each sequence on its own: the same results but for roundings
        gy, gh = c.forward({"seqs": S, "offsets": None}, None, bytes_(fwd))
        for at, seq, (y, hT, _) in parts:
            close(gy.t[at], y, c.d.dtype)
            close(gh[seq], hT)
