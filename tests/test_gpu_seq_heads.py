"""Norm and rotation of the largest heads, in units of every width: pairs, twos, fours and (bf16) eights of angles, up to four units a lane."""
import numpy as np
import pytest
import torch

import paper_1801_04380_amd as sn
import test_gpu_seq
from oracle import seq_oracle as oracle
from test_gpu_seq import SENTINEL, Data, bytes_, close, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 9])
@pytest.mark.parametrize("heads", [(2, 1, 500, 500, False), (1, 1, 500, 252, True), (3, 0, 260, 4, False), (2, 2, 504, 504, True), (1, 1, 512, 256, False), (40, 1, 512, 512, False),
                                   (1, 1, 510, 510, True), (2, 1, 512, 2, False), (40, 2, 268, 8, True)], ids=lambda h: "x".join(map(str, h)))
def test_headnorm(dtype, rows, heads):
    test_gpu_seq.test_headnorm(dtype, rows, heads)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Dh,rot", [(16, 0), (16, 8), (6, 2), (128, 64)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_channels_that_are_not_turned_keep_infinities_to_themselves(dtype, Dh, rot, interleaved):
    """Behind rot_dim no channel has a partner.  An infinite x makes its head's root zero: itself NaN, all others of the head zero.  An infinite dy reaches the
    gradient of its own channel's weight and no other's."""
    d, rows, heads, at = Data(dtype, Dh + rot), 5, 2, Dh + rot + 1          # in the second head
    x, dy = d.normal(rows, heads * Dh), d.normal(rows, heads * Dh)
    freq = (10.0 ** -torch.arange(rot // 2)).float().cuda() if rot else None
    wild = x.clone()
    wild[1, at] = float("inf")
    y, plain = torch.empty_like(x).cuda(), torch.empty_like(x).cuda()
    for v, out in ((x, plain), (wild, y)):
        sn.sn_headnorm_rot_fwd(v.cuda(), None, None, None, None, freq, out, None, Dh, 1e-6, interleaved)
    others = [c for c in range(Dh, 2 * Dh) if c != at]
    assert torch.isnan(y[1, at]) and (y[1, others] == 0).all()
    assert torch.equal(y[[0, 2, 3, 4]], plain[[0, 2, 3, 4]]) and torch.equal(y[1, :Dh], plain[1, :Dh])
    g = dy.clone()
    dw, dx, scratch = torch.full((Dh,), SENTINEL, device="cuda"), torch.empty_like(x).cuda(), bytes_(sn.sn_headnorm_rot_scratch_bytes(rows, heads, 0, Dh))
    g[1, at] = float("inf")
    sn.sn_headnorm_rot_bwd(x.cuda(), None, None, None, None, freq, g.cuda(), None, dx, None, dw, None, scratch, Dh, 1e-6, interleaved)
    _, want = oracle.headnorm_bwd(f64(x), None, np.arange(rows), f64(freq) if rot else np.zeros(0), f64(dy), Dh, 1e-6, interleaved)
    c = at - Dh
    assert dw[c] == float("inf") * float(torch.sign(x[1, at]))
    rest = [i for i in range(Dh) if i != c]
    close(dw[rest], want[rest])
