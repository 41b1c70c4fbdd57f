"""The sequence operators' host side (argument checks, overlaps, sizes) under
AddressSanitizer and UndefinedBehaviorSanitizer: a hipcc build of the host pass only,
as tests/test_sanitizers_cpu.py makes of the other sources."""
import os
import subprocess

import pytest

from test_sanitizers_cpu import HIPCC, ROOT, SAN_ENV, _run


def test_sequence_host_side_under_sanitizers(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    san = "-Xarch_host -fsanitize=address -Xarch_host -fsanitize=undefined".split()
    flags = ["--offload-arch=gfx950", "--offload-host-only", "-O1", "-g", "-std=c++17",
             "-fPIC", *san, *"-Xarch_host -fno-sanitize-recover=all".split(),
             "-I", os.path.join(ROOT, "include")]
    csrc = os.path.join(ROOT, "paper_2301_09266_amd", "csrc")
    srcs = [os.path.join(csrc, f) for f in ("causal_conv.hip", "selective_scan.hip", "add_norm.hip")]
    srcs.append(os.path.join(ROOT, "tests", "sanitize", "sequence_drive.cpp"))
    procs, objs = [], []
    for src in srcs:
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        objs.append(obj)
        procs.append(subprocess.Popen([HIPCC, *flags, "-c", src, "-o", obj],
                                      stderr=subprocess.PIPE, text=True))
    for p in procs:
        err = p.communicate()[1]
        assert p.returncode == 0, err[-4000:]
    exe = str(tmp_path / "sequence_drive")
    subprocess.run([HIPCC, "--offload-arch=gfx950", *san, *objs,
                    "-Wl,--unresolved-symbols=ignore-all", "-o", exe], check=True)
    out = _run(exe, dict(SAN_ENV, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1"))
    assert "all checks held" in out
