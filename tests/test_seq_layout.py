"""CPU: how much memory the scan asks for, by the layout that it picks for sequences of equal length."""
import pytest

import paper_1801_04380_amd as sn


def bytes_of(L, S, channels, states, ragged, dtype=sn.SN_BF16):
    shape = sn.scan_shape(S * L, channels, states, 1, S, dtype, ragged)
    return (sn.sn_scan_states_bytes(shape), sn.sn_scan_workspace_query(shape, sn.SN_SCAN_FWD), sn.sn_scan_workspace_query(shape, sn.SN_SCAN_BWD))


@pytest.mark.parametrize("L", [1, 4, 15, 16, 17, 31, 33, 48, 100])
@pytest.mark.parametrize("channels,states", [(2048, 16), (300, 64), (4096, 5)])
def test_many_sequences_of_few_tiles_take_what_ragged_ones_take(L, channels, states):
    for S in (4096, 65536):
        assert bytes_of(L, S, channels, states, False) == bytes_of(L, S, channels, states, True)


@pytest.mark.parametrize("states", [5, 16, 32, 64])
@pytest.mark.parametrize("S", [1, 3, 64, 700, 4096, 30000])
def test_memory_has_no_step(S, states):
    """One token more a sequence than a whole number of tiles: within 72 MB, or an eighth, of what the same rows take as ragged sequences, kept
    states and the least workspace together."""
    for L in list(range(1, 60)) + [127, 128, 129, 145, 255, 256, 257, 273, 1025]:
        kept, _, (least, _) = bytes_of(L, S, 1536, states, False)
        rkept, _, (rleast, _) = bytes_of(L, S, 1536, states, True)
        assert kept + least <= (rkept + rleast) * 9 / 8 + (72 << 20), L
