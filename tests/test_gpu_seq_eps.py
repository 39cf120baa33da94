"""The norm of heads with the smallest eps."""
import numpy as np
import pytest
import torch

import paper_1801_04380_amd as sn
from oracle import seq_oracle as oracle
from test_gpu_seq import close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("eps", [1e-40, 2.0 ** -149, 1e-38])
def test_eps_below_the_smallest_normal_number(dtype, eps):
    """A head of zeros stays zero, small ones are divided by sqrt(eps) where their squares vanish beside it."""
    Dh = 16
    eps = float(np.float32(eps))
    scale = eps ** 0.5 * 2.0 ** -14                 # squares below 2^-28 of eps
    x = torch.zeros(5, 2 * Dh)
    x[1:, :Dh] = torch.randn(4, Dh, generator=torch.Generator().manual_seed(2)) * scale
    x[3:, Dh:] = 1.5
    x = x.to(dtype)
    y, dx, dy = torch.empty_like(x).cuda(), torch.empty_like(x).cuda(), torch.zeros_like(x)
    sn.sn_headnorm_rot_fwd(x.cuda(), None, None, None, None, None, y, None, Dh, eps)
    want = oracle.headnorm_fwd(x.double().numpy(), None, np.zeros(5), np.zeros(0), Dh, eps, False)
    assert (y[0] == 0).all() and (y[:3, Dh:] == 0).all()
    close(y[1:, :Dh], want[1:, :Dh], dtype)
    close(y[3:, Dh:], want[3:, Dh:], dtype)
    dy[:, 0] = scale
    dy = dy.to(dtype)
    scratch = torch.empty(sn.sn_headnorm_rot_scratch_bytes(5, 2, 0, Dh), dtype=torch.uint8, device="cuda")
    sn.sn_headnorm_rot_bwd(x.cuda(), None, None, None, None, None, dy.cuda(), None, dx, None, None, None, scratch, Dh, eps)
    want, _ = oracle.headnorm_bwd(x.double().numpy(), None, np.zeros(5), np.zeros(0), dy.double().numpy(), Dh, eps, False)
    assert (dx[:, Dh:] == 0).all()
    close(dx[:, :Dh], want[:, :Dh], dtype)
