"""The waits of the 8-bit tile kernels, on the built code (no GPU).

As for the MX4 kernels: LDS transfers complete in the order of issue with every other load, and `s_waitcnt
vmcnt(n)` leaves the n newest outstanding.  The instruction stream of every instance is followed for every length
of the k loop up to a few groups of its four stages: at the wait of stage s the transfers of stage s + 1 must
have landed, however the compiler ordered or dropped the loads between, and no stage's slot is refilled before
its wait."""
import os
import re
import shutil
import subprocess

import pytest

from test_mx4_waits import LIB, OBJDUMP, RING, _between, _parse

GROUP = 4   # stages of the loop


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(OBJDUMP) or not os.path.exists(LIB):
        pytest.skip("the library or llvm-objdump is not there")
    d = tmp_path_factory.mktemp("listing")
    shutil.copy(LIB, d / "l.so")
    subprocess.run([OBJDUMP, "--offloading", "l.so"], cwd=d, check=True, capture_output=True)
    found = {}
    for f in sorted(os.listdir(d)):
        if f.endswith("gfx950"):
            text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", f], cwd=d, check=True, capture_output=True,
                                  text=True).stdout
            for name, body in re.findall(r"^[0-9a-f]+ <(\w*a8_tile_kernel\w*)>:\n(.*?)(?=^\n|\Z)", text, re.S | re.M):
                found[name] = body
    return found


def _check(code, stops, nks):
    """None, or what had not landed.  A wave transfers one piece of each stage."""
    pro, loop, rest, drain = stops[0], stops[1:1 + GROUP], stops[1 + GROUP:2 * GROUP], stops[2 * GROUP]
    route = [pro] + loop * (nks // GROUP) + rest[:nks % GROUP] + [drain]
    states, sent = {()}, 0   # per path: what is outstanding, oldest first; transfers so far
    at = next(i for i, c in enumerate(code) if c and c[0] == "V" and c[1] != "o")
    for n, goal in enumerate(route):
        segments = _between(code, stops, at, goal)
        assert segments, f"no way to the wait of stage {n - 1}"
        moved = {sum(e == ("V", "w") for e in p) for p in segments}
        assert len(moved) == 1
        new = set()
        for queue in states:
            for p in segments:
                q, k = list(queue), sent
                for kind, v in p + (code[goal],):
                    if kind == "wait":
                        q = q[max(0, len(q) - v):] if v else []
                    elif v == "o":
                        q.append(-1)
                    else:
                        q.append(k)
                        k += 1
                new.add(tuple(q))
        states, sent = new, sent + moved.pop()
        assert len(states) <= 64
        if goal == drain:
            return None if all(not q for q in states) else "the drain"
        s = n - 1   # the stage whose wait this is (-1: the prologue's, for stage 0)
        assert sent <= s + RING + 1
        if s + 1 < nks and any(0 <= j <= s + 1 for q in states for j in q):
            return f"stage {s + 1} at the wait of stage {s}"
        at = goal + 2


def test_every_stage_has_landed_when_it_is_read(kernels):
    assert len(kernels) == 36   # two weight formats, two widths, three activations, three types
    bad = []
    for name, body in kernels.items():
        code, stops = _parse(body)
        assert len(stops) == 2 * GROUP + 3, f"{name}: {len(stops)} waits, not the prologue's, 4 + 3 stages' and three behind them"
        for nks in range(1, 14):
            r = _check(code, stops, nks)
            if r:
                bad.append((name, nks, r))
    assert not bad, f"{len(bad)} of them, the first: {bad[:3]}"


def test_the_check_finds_a_wait_that_is_too_loose(kernels):
    """The same with a count one transfer and two loads higher, in the listing."""
    name, body = next(iter(kernels.items()))
    code, stops = _parse(body)
    i = stops[2]
    code[i] = ("wait", code[i][1] + 3)
    assert _check(code, stops, 8) == "stage 2 at the wait of stage 1"
