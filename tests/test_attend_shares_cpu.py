"""Which states the launches of linear attention over shares read and write, where the result lies in the state that the
call was given: workgroups of one launch run in no order, so none may read what another writes.  The rules are those
that the kernels include (csrc/attend_shares.h), built here for the host."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1810_08061_amd", "csrc")
NOTHING, GIVEN, SLOT = range(3)

SOURCE = """
#include "attend_shares.h"
extern "C" int used(int L, int span) { return ldyn::shares_used(L, span); }
extern "C" int ends(int share, int used, int back) { return ldyn::ends_row(share, used, back); }
extern "C" int adds(int share, int used, int back) { return ldyn::adds(share, used, back); }
extern "C" int start(int share, int used) { return (int)ldyn::start_of(share, used); }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    at = tmp_path_factory.mktemp("shares")
    (at / "rules.cpp").write_text(SOURCE)
    out = str(at / "rules.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(at / "rules.cpp"), "-o", out], check=True)
    return ctypes.CDLL(out)


def _launches(rules, L, span, shares, back):
    """A row's launches as lists of workgroups, each (buffers read, buffers written); the result is the given state itself."""
    used = rules.used(L, span)
    slots = [("slot", s) for s in range(used)]
    states = [(set(), {("slot", s)}) for s in range(shares) if rules.adds(s, used, back)]
    # one thread of the join has an element of the given state and of all slots to itself
    join = [({"given", *slots}, set(slots))] if used > 1 else []
    passes = []
    for s in range(shares):
        start = rules.start(s, used)
        passes.append(({GIVEN: {"given"}, SLOT: {("slot", s)}, NOTHING: set()}[start], {"given"} if rules.ends(s, used, back) else set()))
    return used, [states, join, passes]


@pytest.mark.parametrize("back", [0, 1])
def test_no_workgroup_reads_what_another_of_its_launch_writes(rules, back):
    for span in (32, 64, 128, 1024):
        for shares in (1, 2, 3, 8):
            for L in {0, 1, span - 1, span, span + 1, (shares - 1) * span, (shares - 1) * span + 1, shares * span}:
                if L > shares * span:
                    continue
                used, launches = _launches(rules, L, span, shares, back)
                assert 1 <= used <= shares and used == max(1, -(-L // span))
                for launch in launches:
                    for i, (_, written) in enumerate(launch):
                        for j, (read, also) in enumerate(launch):
                            assert i == j or not written & (read | also), (span, shares, L, i, j)
                states, _, passes = launches
                # every share but the one that ends the row leaves its sum; one share leaves the result; each that has steps
                # starts from a state
                assert len(states) == used - 1 and sum(bool(w) for _, w in passes) == 1
                assert [bool(r) for r, _ in passes] == [s < used for s in range(shares)]


def test_the_kernels_go_by_these_rules():
    with open(os.path.join(CSRC, "attend.hip")) as f:
        source = re.sub(r"//[^\n]*", "", f.read())
    body = source[source.index("attend_kernel(AttendParams p)"):source.index("attend_join_kernel(AttendParams p)")]
    given = [line for line in body.splitlines() if "a.start" in line]
    assert len(given) == 1 and "Start::GIVEN" in given[0] and "start_of(share, used)" in body
    assert "ends_row(share, used, a.back)" in body and "adds(share, used, a.back)" in body
