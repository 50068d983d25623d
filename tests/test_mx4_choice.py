"""The choices that products of 4-bit rows make by their sizes, on the CPU: the
header that makes them is plain C++ and is compiled here with g++."""

import os
import shutil
import subprocess

import numpy as np
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
        text = "".join(f"{what} " + " ".join(map(str, (*s, 0, 0, 0, 0, 0)[:6])) + "\n" for s in sizes)
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


def test_height_of_tiles_by_the_parts_that_are_launched(ask):
    """Of 128 and 256 rows what takes less time by the model of the header, a round of 256
    workgroups at a time, with the parts of the sum that the launch really has."""
    # measured, us with 256 and 128 rows: 38, 27; 37, 26; 30, 22; 32, 22; 31, 27; gradients 36, 29; 32, 27
    sizes = [(2, 256, 32000, 1024, 0), (2, 256, 20000, 1024, 0), (2, 256, 30000, 768, 0), (2, 500, 16000, 768, 0),
             (1, 161, 5818, 1024, 0), (1, 670, 734, 2048, 1), (2, 1240, 1895, 384, 1)]
    assert [t for t, _ in ask("gemm", sizes)] == [128] * len(sizes)
    rng = np.random.default_rng(0)
    for back in (0, 1):
        m, n, d = (np.exp(rng.uniform(np.log(lo), np.log(hi), 500)).astype(int) for lo, hi in ((129, 4000), (64, 200000), (33, 5000)))
        sizes = [(int(i % 3), int(a), int(b), int(c), back) for i, (a, b, c) in enumerate(zip(m, n, d))]
        parts = {h: [p for p, in ask("parts", [(*s, h) for s in sizes])] for h in (128, 256)}
        for i, (s, (chosen, p)) in enumerate(zip(sizes, ask("gemm", sizes))):
            cols, length = (s[3], s[2]) if back else (s[2], s[3])
            time = {}
            for h, cost in ((128, 5), (256, 8)):
                groups, tiles = -(-length // 128), -(-cols // 256) * -(-s[1] // h)
                time[h] = cost * -(-tiles * parts[h][i] // 256) * -(-groups // parts[h][i])
            assert chosen == (128 if time[128] < time[256] else 256) and p == parts[chosen][i], (s, time)


def test_gpu_tests_reach_every_arrangement(ask):
    """The sizes of test_gpu_mx4_tiles.py take every height of tiles of each direction, in one
    part and in several, and every form of 4-bit by 4-bit: a rule that changes fails here."""
    pytest.importorskip("torch")
    from tests import test_gpu_mx4_tiles as T

    for type_ in (0, 1, 2):
        score = ask("gemm", [(type_, *s, 0) for s in T.SCORE])
        assert {t for t, _ in score} == {0, 16, 32, 64, 128, 256}
        back = ask("gemm", [(type_, *s, 1) for s in T.BACKWARD])
        assert {t for t, _ in back} == {16, 32, 64, 128, 256}
        for got in (score, back):
            assert {(t, p > 1) for t, p in got if t >= 64} == {(t, p) for t in (64, 128, 256) for p in (False, True)}, got
        # 256 rows with odd and even numbers of groups in a part
        for sizes, got, length in ((T.SCORE, score, 2), (T.BACKWARD, back, 1)):
            per = [-(-(-(-s[length] // 128)) // p) for s, (t, p) in zip(sizes, got) if t == 256]
            assert {v % 2 for v in per} == {0, 1} and max(per) >= 5
    forms = {}
    for (m, n, dim, _), (side, _, _) in zip(T.MATMUL, ask("form", [s[:2] for s in T.MATMUL])):
        forms.setdefault(side, set()).add(-(-dim // 128))
    assert set(forms) == {256, 128, 64, 32, 16}
    assert {5, 6, 8, 9} <= forms[256] and max(forms[128]) >= 9
