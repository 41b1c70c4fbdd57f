"""What the sequence operators launch, without a GPU (tests/sequence_launch_drive.cpp
stands in for the HIP runtime): every size that the header promises is one the
device takes, with a workgroup for all of its work."""
import os
import subprocess

import pytest

from paper_2301_09266_amd import finc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
LDS = 160 * 1024


@pytest.fixture(scope="module")
def drive(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    exe = str(tmp_path_factory.mktemp("drive") / "sequence_launch_drive")
    subprocess.run([HIPCC, "--offload-host-only", "-x", "c++", "-std=c++17", "-O1", "-rdynamic",
                    "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                    "-D__HIP_PLATFORM_AMD__",
                    os.path.join(ROOT, "tests", "sequence_launch_drive.cpp"), "-ldl", "-o", exe],
                   check=True)

    def run(calls):
        """[(op, type, B, D, L, N, G)] -> [(rc, [(kernel, blocks, threads, lds)])]"""
        text = "".join(" ".join(map(str, c)) + "\n" for c in calls)
        r = subprocess.run([exe, finc.LIB_PATH], input=text, capture_output=True, text=True,
                           timeout=120)
        assert r.returncode == 0, r.stderr
        out = []
        for line in r.stdout.splitlines():
            rc, *ls = line.split(";")
            got = []
            for x in ls:
                name, *n = x.rsplit(",", 5)
                gx, gy, gz, threads, lds = map(int, n)
                assert gx * threads < 2**32 and 0 < gy < 2**16 and 0 < gz < 2**16, (line, calls)
                assert 0 < threads <= 1024 and lds <= LDS, line
                got.append((name, gx * gy * gz, threads, lds))
            out.append((int(rc), got))
        assert len(out) == len(calls)
        return out
    return run


def up(a, b):
    return -(-a // b)


F32, BF16 = finc.F32, finc.BF16
MANY = (1 << 31) - 300
# (call, the least workgroups of its first kernel)
WIDE = [
    # rows of positions that fill half of their lanes or less: a workgroup's rows, its tiles
    (("conv", BF16, 1 << 15, 1 << 15, 17, 4, 0), (1 << 30) // 64),
    (("conv", BF16, 1 << 13, 1 << 10, 2049, 4, 0), (1 << 23) * 2),
    (("conv", F32, 1, MANY, 5, 1, 0), up(MANY, 128)),
    (("conv", BF16, 1, MANY, 1, 1, 0), up(MANY, 256)),
    # a workgroup a channel
    (("conv_back", BF16, 1, 1 << 24, 1, 4, 0), 1 << 24),
    (("conv_back", F32, 3, (1 << 24) + 7, 40, 8, 0), (1 << 24) + 7),
    (("conv_back", BF16, 1, MANY, 1, 1, 0), MANY),
    (("conv_step", BF16, 1, MANY, 1, 8, 0), up(MANY, 256)),
    # eight channels of a group a workgroup, 64 in a short raster
    (("scan", BF16, 1 << 13, 1 << 10, 65, 1, 1 << 10), 1 << 23),
    (("scan", F32, 1 << 20, 1 << 10, 130, 16, 1), 1 << 27),
    (("scan", BF16, 1 << 16, 1 << 14, 65, 1, 1 << 14), 1 << 30),
    (("scan", BF16, 1 << 14, 1 << 10, 1, 1, 1 << 10), 1 << 24),
    (("scan", BF16, 1 << 16, 1 << 14, 64, 2, 1 << 13), 1 << 29),
    (("scan_back", BF16, 1 << 13, 1 << 10, 65, 1, 1 << 10), 1 << 23),
    (("scan_back", BF16, 1 << 14, 16, 64, 32, 16), 1 << 18),    # 2^24 rows of dB and dC
    (("scan_back", BF16, 1 << 14, 1 << 10, 1, 64, 1 << 10), 1 << 24),   # and 2^31
    (("scan_back", F32, 1, 1 << 23, 1, 62, 1), 1 << 17),        # 2^24 workgroups' parameters
    (("scan_back", F32, 1, 1 << 26, 1, 64, 1), 1 << 20),
    (("scan_step", F32, 1, 1 << 30, 1, 5, 1), 1),
    (("scan_step", BF16, 1, MANY, 1, 1, 1), 1),
    (("norm", BF16, 1 << 30, 8, 0, 0, 0), 1), (("norm8", BF16, 1 << 30, 8, 0, 0, 0), 1),
    (("norm_back", BF16, 1 << 30, 8, 0, 0, 0), 1), (("dropout", F32, 1 << 30, 8, 0, 0, 0), 1),
    (("norm", F32, 1 << 19, 16384, 0, 0, 0), 1), (("norm_back", F32, 1 << 19, 16384, 0, 0, 0), 1),
]


@pytest.mark.parametrize("call,least", WIDE)
def test_many_rows_are_launched(drive, call, least):
    (rc, ls), = drive([call])
    assert rc == finc.OK and ls, (call, rc, ls)
    assert ls[0][1] >= least, (call, ls)


def test_ordinary_calls_take_one_row_of_workgroups(drive):
    """No more workgroups than the work."""
    calls = [(("conv", F32, 64, 512, 256, 4, 0), 64 * 512 // 4),
             (("conv_back", BF16, 8, 2048, 4096, 4, 0), 2048),
             (("scan", BF16, 1, 2048, 4096, 16, 1), 256),
             (("scan", BF16, 64, 2048, 16, 16, 1), 64 * 32),
             (("scan_back", BF16, 4, 2048, 4096, 16, 1), 256),
             (("scan_step", F32, 100, 1024, 1, 16, 1), 100 * 16)]
    for (call, want), (rc, ls) in zip(calls, drive([c for c, _ in calls])):
        assert rc == finc.OK and ls[0][1] == want, (call, ls)
    # dB and dC: a workgroup for 1024 positions of a row; the parameters: for 32 of them
    (_, ls), = drive([calls[4][0]])
    assert [blocks for _, blocks, _, _ in ls[1:]] == [2 * 4 * 16 * 4, 2048 * 18 // 32]


@pytest.mark.parametrize("S,D,N", [(1 << 30, 1 << 30, 16), (1 << 30, 1 << 30, 64),
                                   ((1 << 31) - 1, 1 << 30, 9), (1 << 28, 1 << 30, 64)])
def test_states_past_the_address_space_are_refused(S, D, N):
    """Entries whose number would wrap to a small one."""
    at = [1 << (40 + i) for i in range(10)]
    a = finc.SCAN_STEP_ARGS.pack(BF16, 1, S, D, N, 1, 1, at[0], at[1], 0, at[2], at[3], D, D, D,
                                 N, N, D, at[4], at[5], 0, 0, 0, 0)
    assert finc.lib().finc_selective_scan_step(a, None) == finc.EINVAL
    assert finc.lib().finc_causal_conv_step(BF16, at[0], D, at[1], D, at[2], None, None, None, 1,
                                            S, D, 8, 1, None) == finc.EINVAL
