"""CPU: what the token-sequence layers launch (tests/launches/seq_recorder.cpp): every kernel of theirs that is in the library is reached by some call,
and no call asks for a grid beyond what the hardware takes."""
import os
import re
import subprocess

import pytest

from paper_1801_04380_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.join(ROOT, "tests", "launches")


@pytest.fixture(scope="module")
def lines():
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    exe = os.path.join(HERE, "_build", "seq_recorder")
    _lib.load()
    subprocess.run(["g++", "-O1", "-std=c++17", "-rdynamic", "-I", os.path.join(ROOT, "include"), "-o", exe, os.path.join(HERE, "seq_recorder.cpp"),
                    _lib.LIB_PATH, "-Wl,-rpath," + os.path.dirname(_lib.LIB_PATH), "-Wl,--allow-shlib-undefined"], check=True)
    env = dict(os.environ, LD_LIBRARY_PATH="/opt/rocm/lib:" + os.environ.get("LD_LIBRARY_PATH", ""))
    out = subprocess.run([exe], stdout=subprocess.PIPE, text=True, check=True, env=env).stdout
    return [line.split(" ", 1) for line in out.splitlines()]


def test_every_kernel_is_reached(lines):
    assert [what for kind, what in lines if kind == "bad"] == []
    ours = re.compile(r"_ZN2sn12_GLOBAL__N_1\d+(conv1d_(fwd|bwd|dstate|sum|step)|headnorm(_sum)?|scan_(fwd|bwd|bwd_local|carry|join|step))_kernel")
    has = {what for kind, what in lines if kind == "has" and ours.match(what)}
    launched = {what for kind, what in lines if kind == "launched"}
    assert len(has) > 250 and launched <= has
    assert sorted(has - launched) == []


def test_empty_sequences_are_shared_out(lines):
    """800 rows in 4096 sequences, 2048 channels: whoever hands on the states of the empty ones has no more than 16 sequences of a block of channels."""
    grids = dict(what.rsplit(" ", 1) for kind, what in lines if kind == "grid")
    for kernel in ("conv1d_fwd_kernel", "scan_fwd_kernel", "scan_join_kernel"):
        found = [int(n) for name, n in grids.items() if kernel in name]
        assert found and max(found) > 4096 // 16
