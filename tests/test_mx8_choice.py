"""The arrangements that products of 8-bit rows with 4-bit rows choose by their sizes, on
the CPU: the header that chooses is plain C++ and is compiled here with g++."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FEW, TILE256, TILE = 0, 1, 2
MOST_ROWS = 0x7FFFFF00


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("mx8_choice") / "driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2608_30384_amd", "csrc"),
                    os.path.join(ROOT, "tests", "mx8_choice_driver.cpp"), "-o", exe], check=True)

    def ask(sizes):
        r = subprocess.run([exe], input="".join("%d %d %d %d\n" % s for s in sizes), capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        return [tuple(map(int, line.split())) for line in r.stdout.splitlines()]

    return ask


def test_forms(ask):
    sizes = [(m, n, steps, exact) for m in (1, 16, 17, 64, 65, 255, 256, 4096, 65535 * 64) for n in (1, 64, 4096, 100_003, MOST_ROWS)
             for steps in (1, 3, 4, 11, 12, 512) for exact in (0, 1)]
    for (m, n, steps, exact), (form, split, held) in zip(sizes, ask(sizes)):
        blocks = -(-m // 16) * -(-n // 16)
        assert (form == FEW) == (m <= 16 or blocks <= (3500 if exact else 2000))
        if form == TILE256:
            tiles = -(-m // 256) * -(-n // 256)
            assert tiles >= 256 and steps >= 12
        if form == FEW:
            # every wavefront has a group where they are shared out, and a's codes and scales
            # fit beside the joined sums in half of a CU's LDS
            assert not split or steps >= 4
            assert not held or min(m, 16) * steps * 132 + 4096 <= 80 * 1024


def test_measured_sizes(ask):
    got = ask([(1, 131072, 6, 1), (1, 4096, 32, 1), (255, 100_003, 8, 1), (8192, 32768, 32, 0), (300, 100_000, 6, 0),
               (16, 4096, 32, 1), (16, 4096, 33, 1), (64, 1000, 32, 0), (64, 16_000, 12, 0), (64, 16_000, 12, 1),
               (128, 4000, 6, 1)])
    assert [g[0] for g in got] == [FEW, FEW, TILE, TILE256, TILE, FEW, FEW, FEW, TILE, TILE, FEW]
    assert [g[1] for g in got[:2]] == [0, 1] and [g[2] for g in got[5:7]] == [1, 0]
