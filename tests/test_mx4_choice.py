"""The choices that products of 4-bit rows make by their sizes, on the CPU: the
header that makes them is plain C++ and is compiled here with g++."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MOST_ROWS = 0x7FFFFF00
MOST_M = 65535 * 64


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("mx4_choice") / "driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2608_30384_amd", "csrc"),
                    os.path.join(ROOT, "tests", "mx4_choice_driver.cpp"), "-o", exe], check=True)

    def ask(what, sizes):
        text = "".join(f"{what} " + " ".join(map(str, s)) + "\n" for s in sizes)
        r = subprocess.run([exe], input=text, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        out = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
        assert len(out) == len(sizes)
        return out

    return ask


def test_direct_grids_hold_their_threads(ask):
    """A launch counts the threads along x in 32 bits and the workgroups along y in 16."""
    ns = [1, 63, 64, 65, 4096, 100_003, (1 << 30) - 64, (1 << 30) - 63, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, MOST_ROWS]
    ms = [1, 15, 16, 17, 32, 33, 64, 65, 1000, 65536, MOST_M - 1, MOST_M]
    for n in ns:
        for m, (side, x, y) in zip(ms, ask("form", [(m, n) for m in ms])):
            if side < 128:
                assert x * 256 < 1 << 32 and y <= 65535, (m, n, side, x, y)
                assert x * 4 * side >= n and y * side >= m


def test_rows_of_the_longest_sums(ask):
    """The slabs that the gradient asks for run up to eight past its last group: none
    comes out as a row inside the sum (nor, as a 32-bit number that has wrapped, below it)."""
    for rows in (1, 128, 129, MOST_ROWS // 2, MOST_ROWS - 511, MOST_ROWS - 1, MOST_ROWS):
        groups = -(-rows // 128)
        slabs = range(max(0, 4 * groups - 9), 4 * groups + 9)
        for own in (0, 31):
            for slab, (row,) in zip(slabs, ask("slab_row", [(own, s) for s in slabs])):
                assert row == own + 32 * slab
