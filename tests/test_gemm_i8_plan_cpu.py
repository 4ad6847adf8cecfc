"""Products of 8-bit integers, the choice of their kernels: the shapes of the GPU tests run the kernels that they are listed for, none is left out, and parts of k are ones that the
kernels and the workspace hold."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2006_06762_amd", "csrc")


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    """(tile's edges, buffers, parts of k) or (blocks of sixteen rows, waves) for each of a list of (M, N, K)."""
    where = tmp_path_factory.mktemp("i8")
    (where / "choose.cpp").write_text("""
#include <cstdio>
#include "gemm_i8_plan.h"
using namespace anr::i8;
int main()
{
    const int buffers[TILES] = {2, 2, 3, 3, 3, 4};
    long M, N, K;
    printf("%d\\n", (int)TILES);
    while (scanf("%ld %ld %ld", &M, &N, &K) == 3) {
        const Choice c = choose(M, N, K);
        const int blocks = (int)(M + 15) / 16;
        if (c.tile == ROWS) printf("rows %d %d\\n", blocks, waves_of(N, K, most_waves(blocks)));
        else printf("tile %d %d %d %d\\n", kShapes[c.tile].m, kShapes[c.tile].n, buffers[c.tile], c.splits);
    }
}
""")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-O2", "-I", CSRC, str(where / "choose.cpp"), "-o", str(where / "choose")], check=True)

    def of(shapes):
        out = subprocess.run([str(where / "choose")], input="\n".join("%d %d %d" % s for s in shapes), capture_output=True, text=True, check=True).stdout.split("\n")
        return int(out[0]), [(kind, *map(int, rest)) for kind, *rest in (line.split() for line in out[1:] if line)]
    return of


def test_shapes_of_the_gpu_tests_run_what_they_are_listed_for(choose):
    gpu = pytest.importorskip("test_gemm_i8_kernels_gpu")
    around = lambda s: [(s[0], n, k) for n in (s[1], s[1] + 3) for k in (s[2], s[2] + 1)]  # noqa: E731
    tiles, _ = choose([])
    assert len(gpu.TILED) == 2 * tiles and {b for b, _ in gpu.ROWS} == {1, 2, 3, 4}
    for (m, n, buffers, shared), shape in gpu.TILED.items():
        assert shape[1] % 64 == 0 and shape[2] % 4 == 0 and shape[2] % 128 not in (0, 127)
        for got in choose(around(shape))[1]:
            assert got[:4] == ("tile", m, n, buffers) and (got[4] > 1) == shared, (shape, got)
    for kernel, shape in gpu.ROWS.items():
        for got in choose(around(shape))[1]:
            assert got == ("rows", *kernel), (shape, got)


def test_parts_of_k(choose):
    """At least four chunks of 128 in each part, sixteen parts at most; few rows are 64 at most, by waves whose two buffers each fit
    a CU's LDS."""
    shapes = [(M, N, K) for M in (1, 16, 17, 33, 64, 65, 300, 5000, 100000, (1 << 22) - 1) for N in (1, 63, 1024, 4100, 20000, 1 << 20) for K in (1, 128, 513, 4096, 11264, (1 << 17) - 1)]
    for (M, N, K), (kind, *c) in zip(shapes, choose(shapes)[1]):
        if kind == "rows":
            assert M <= 64 and c[0] == (M + 15) // 16 and c[1] in (4, 8, 16) and c[1] * 2 * (16 * (1 + c[0]) * 128 + 512) <= 160 << 10
            continue
        m, n, _, parts = c
        assert 1 <= parts <= 16 and (parts == 1 or (K + 127) // 128 // parts >= 4)
        # (a grid has fewer than 2^32 threads, for results that the card's memory holds)
        if M * N * 2 <= 288 << 30:
            assert -(-M // m) * -(-N // n) * parts * (512 if m == 256 else 256) < 1 << 32
