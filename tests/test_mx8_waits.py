"""Counted waits of the 8-bit by 4-bit products' tiles, in the built library's own code.

k_mx8_score_tile and k_mx8_score_tile_f32 have a group's codes and scales written to LDS by
the memory unit while the group before is multiplied.  Where the loads of the group after
are out too, `s_waitcnt vmcnt(N)` waits for all but the N last operations, N the loads of a
group: that is a wait for the next group only if the N loads after its last one come before
the wait.  In the assembly of the kernels built from this tree, between a counted wait and
the last jump or label before it there have to be N loads to LDS or more.
"""

import re

from .test_mx4_waits import functions, is_load_to_lds, library  # noqa: F401


def counted_waits(code):
    """Of each counted wait ahead of a barrier: its N, and the loads to LDS since the last jump or label."""
    waits, loads = [], 0
    for i, at in enumerate(code):
        if is_load_to_lds(at):
            loads += 1
        elif at.startswith("s_cbranch") or at.startswith("s_branch") or at.endswith(">:"):
            loads = 0
        m = re.match(r"s_waitcnt .*vmcnt\((\d+)\)", at)
        if m and int(m.group(1)) and code[i + 1].startswith("s_barrier"):
            waits.append((int(m.group(1)), loads))
    return waits


def test_loads_of_the_group_after(library, tmp_path):  # noqa: F811
    kernels = functions(library, "k_mx8_score_tile", tmp_path)
    kernels = {k: v for k, v in kernels.items() if not k.endswith(".kd")}
    assert len(kernels) == 6        # two heights of tiles to float16, to bfloat16 and to float32
    in_loop = 0
    for name, code in kernels.items():
        waits = counted_waits(code)
        # ahead of the loop those of two groups; in it, with three places for a group, those of one
        assert waits and waits[0][1] >= 2 * waits[0][0], name
        for n, loads in waits[1:]:
            in_loop += 1
            assert n == waits[0][0] and loads >= n, (name, n, loads)
    assert in_loop >= 2             # tiles of 256 rows to either 16-bit type


def test_the_count_itself():
    lds, wait = "buffer_load_dwordx4 v0, s[0:3], 0 offen lds", "s_waitcnt vmcnt(2) lgkmcnt(0)"
    assert counted_waits([lds, lds, wait, "s_barrier"]) == [(2, 2)]
    assert counted_waits([lds, "<L1>:", lds, wait, "s_barrier"]) == [(2, 1)]
    assert counted_waits([lds, lds, "s_waitcnt vmcnt(0)", "s_barrier"]) == []
