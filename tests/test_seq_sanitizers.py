"""AddressSanitizer + UndefinedBehaviorSanitizer builds of the token-sequence layers' CPU-side code: how the kernels walk along packed rows
(csrc/seq_walk.h, tests/sanitize/seq_walk_driver.cpp), and the host side of their calls over sizes of all kinds
(csrc/seq*.hip without their kernels, tests/launches/seq_recorder.cpp).  Nothing here launches a kernel or needs a GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1801_04380_amd", "csrc")
OUT = os.path.join(ROOT, "tests", "sanitize", "_build")
ENV = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")


def _run(cmd, **kw):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, **kw)
    assert r.returncode == 0, "%s\n%s" % (" ".join(cmd), r.stdout[-4000:])
    return r.stdout


def test_walk_along_packed_rows():
    os.makedirs(OUT, exist_ok=True)
    exe = os.path.join(OUT, "seq_walk_driver")
    _run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-omit-frame-pointer", "-fno-sanitize-recover=undefined", "-I", CSRC, "-o", exe,
          os.path.join(ROOT, "tests", "sanitize", "seq_walk_driver.cpp")])
    assert "walk driver: ok" in _run([exe], env=ENV)


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc builds the host side of the .hip sources")
def test_host_side_of_the_calls():
    from paper_1801_04380_amd import build
    os.makedirs(OUT, exist_ok=True)
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-Xarch_host", "-fno-omit-frame-pointer"]
    objs = []
    for name in ("seq_api", "seq_conv1d", "seq_headnorm", "seq_scan", "seq_scan_bwd"):
        objs.append(os.path.join(OUT, name + ".host.o"))
        _run(["hipcc", "--offload-host-only"] + [f for f in build.FLAGS if f != "-O3"] + ["-O1", "-g", "-w"] + san +
             ["-c", os.path.join(CSRC, name + ".hip"), "-o", objs[-1]])
    exe = os.path.join(OUT, "seq_host_driver")
    drv = os.path.join(OUT, "seq_recorder.o")
    _run(["hipcc", "--offload-host-only", "-O1", "-g", "-std=c++17", "-I", os.path.join(ROOT, "include")] + san +
         ["-c", os.path.join(ROOT, "tests", "launches", "seq_recorder.cpp"), "-o", drv])
    # the kernels' code is left out, and the symbols that stand for it with it
    _run(["hipcc", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize", "-Wl,--unresolved-symbols=ignore-all", "-o", exe, drv] + objs)
    out = _run([exe], env=ENV)
    assert "bad" not in out and out.count("launched") >= 1
