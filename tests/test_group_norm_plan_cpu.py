"""How the group norm divides its calls, on the CPU with the kernels' own arithmetic."""
import os
import subprocess

import pytest

from test_gemm_plan_cpu import CSRC, HERE


@pytest.fixture(scope="module")
def lds(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("norm") / "lds")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-I", CSRC, os.path.join(HERE, "group_norm_lds.cpp"), "-o", exe], check=True)
    return lambda lines: subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True)


def test_work_groups_use_the_shared_memory_that_their_launch_asks_for(lds):
    """Groups of every width below 400 in such numbers that the last chunk is any part of a full one, few and many images (a work-group
    that holds its chunk, one that does not), and the widest groups that a call takes."""
    lines = []
    for cg in list(range(1, 400)) + [500, 1000, 1023, 1024, 2047, 2560, 4095, 4096, 8190, 8191, 8192]:
        per = max(1, -(-64 // cg))                  # groups of a chunk, at most
        for groups in sorted({*range(1, min(2 * per, 24) + 2), 24, 32, 40}):
            C = cg * groups
            for es in (2, 4):
                for vector in (0, 1):
                    for N, HW in ((1, 49), (2, 400), (3, 5), (4, 5985), (300, 64)):
                        lines += ["%d %d %d %d %d %d %d" % (N, HW, C, groups, es, vector, b) for b in (0, 1)]
    res = lds(lines)
    assert res.returncode == 0, res.stdout[-4000:]
    assert int(res.stdout) > 1000                   # calls whose last chunk uses more than a full one are among them
