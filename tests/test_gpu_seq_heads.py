"""Norm and rotation of the largest heads, in units of every width: pairs, twos, fours and (bf16) eights of angles, up to four units a lane."""
import pytest

import test_gpu_seq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 9])
@pytest.mark.parametrize("heads", [(2, 1, 500, 500, False), (1, 1, 500, 252, True), (3, 0, 260, 4, False), (2, 2, 504, 504, True), (1, 1, 512, 256, False), (40, 1, 512, 512, False),
                                   (1, 1, 510, 510, True), (2, 1, 512, 2, False), (40, 2, 268, 8, True)], ids=lambda h: "x".join(map(str, h)))
def test_headnorm(dtype, rows, heads):
    test_gpu_seq.test_headnorm(dtype, rows, heads)
