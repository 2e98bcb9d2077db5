"""The waits of the MX4 tile kernels, on the built code (no GPU).

The tile kernels' LDS transfers complete in the order of issue with every other load, and
`s_waitcnt vmcnt(n)` leaves the n newest outstanding.  Here the instruction stream of every
instance is followed for every length of the k loop: at the wait of stage s the transfers of
stage s + 1 must have landed, and at the last stage of a quad the scales of the next one, however
the compiler ordered or dropped the loads between.
"""
import os
import re
import shutil
import subprocess

import pytest

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_24416_amd", "libclq.so")
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
RING = 5   # stages of channel units in flight


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
            for name, body in re.findall(r"^[0-9a-f]+ <(\w*mx_tile_kernel\w*)>:\n(.*?)(?=^\n|\Z)", text, re.S | re.M):
                found[name] = body
    return found


def _parse(body):
    """[(kind, value)] by address order: V (a load or store; "w" or "s" for a transfer of codes
    or scales), wait, jump, branch, end; and the waits with a barrier behind them."""
    lines = []
    for text, addr in re.findall(r"^\t(.*?)\s*// ([0-9A-F]+):", body, re.M):
        lines.append((int(addr, 16), text))
    at = {a: i for i, (a, _) in enumerate(lines)}
    code, stops = [], []
    for i, (a, t) in enumerate(lines):
        op = t.split()[0]
        if op == "s_waitcnt":
            n = re.search(r"vmcnt\((\d+)\)", t)
            code.append(("wait", int(n[1]) if n else None))
            if "lgkmcnt(0)" in t and i + 1 < len(lines) and lines[i + 1][1].split()[0] == "s_barrier":
                stops.append(i)
        elif op == "s_branch" or op.startswith("s_cbranch"):
            off = int(t.split()[1])
            off -= 65536 if off >= 32768 else 0
            code.append(("jump" if op == "s_branch" else "branch", at[a + 4 + 4 * off]))
        elif op == "s_endpgm":
            code.append(("end", None))
        elif re.match(r"(buffer|global|flat|scratch)_(load|store|atomic)", op):
            code.append(("V", ("w" if "dwordx4" in op else "s") if t.split()[-1] == "lds" else "o"))
        else:
            code.append(None)
    return code, stops


def _between(code, stops, start, goal):
    """The events of every path from instruction `start` to stop `goal` that meets no other."""
    stop, paths, work, seen = set(stops), set(), [(start, ())], set()
    while work:
        i, ev = work.pop()
        while (i, ev) not in seen:
            assert len(ev) < 200, "a loop between two waits"
            if code[i] and code[i][0] != "V":
                seen.add((i, ev))
            if i in stop:
                if i == goal:
                    paths.add(ev)
                break
            c = code[i]
            if c is None or c == ("wait", None):
                i += 1
            elif c[0] == "end":
                break
            elif c[0] == "jump":
                i = c[1]
            elif c[0] == "branch":
                work.append((c[1], ev))
                i += 1
            else:
                ev += (c,)
                i += 1
    return paths


def _check(code, stops, per_wave, nks):
    """None, or what had not landed."""
    pro, loop, last, drain = stops[0], stops[1:9], stops[9:16], stops[16]
    route = [pro] + loop * (nks // 8) + last[:nks % 8] + [drain]
    states = {()}   # per path: kinds outstanding, oldest first, as (kind, index)
    # (what was loaded ahead of the first transfer lands before it)
    at = next(i for i, c in enumerate(code) if c and c[0] == "V" and c[1] != "o")
    count = {"w": 0, "s": 0}
    for n, goal in enumerate(route):
        segments = _between(code, stops, at, goal)
        assert segments, f"no way to the wait of stage {n - 1}"
        assert len({tuple(e for e in p if e[0] == "V" and e[1] != "o") for p in segments}) == 1
        new, counts = set(), None
        for queue in states:
            for p in segments:
                q, c = list(queue), dict(count)
                for kind, v in p + (code[goal],):
                    if kind == "wait":
                        q = q[max(0, len(q) - v):]
                    elif v == "o":
                        q.append(("o", 0))
                    else:
                        q.append((v, c[v] // per_wave))
                        c[v] += 1
                counts = c
                new.add(tuple(q))
        states, count = new, counts
        if goal == drain:
            break
        s = n - 1   # the stage whose wait this is (-1: the prologue's, for stage 0)
        assert count["w"] // per_wave <= s + RING + 1
        for q in states:
            if s + 1 < nks:
                if any(k == "w" and j <= s + 1 for k, j in q):
                    return f"stage {s + 1}'s channel units at the wait of stage {s}"
                if (s + 1) % 4 == 0 and any(k == "s" and j <= (s + 1) // 4 for k, j in q):
                    return f"quad {(s + 1) // 4}'s scales at the wait of stage {s}"
        # (only what is outstanding at the newest wait matters further on)
        assert len(states) <= 64
        at = goal + 2
    return None


def test_every_stage_has_landed_when_it_is_read(kernels):
    assert len(kernels) > 20
    bad = []
    for name, body in kernels.items():
        code, stops = _parse(body)
        assert len(stops) == 18, f"{name}: {len(stops)} waits, not the prologue's, 8 + 7 stages' and two at the end"
        per_wave = 4 // int(re.search(r"mx_tile_kernelILi(\d)", name)[1])
        for nks in range(1, 25):
            r = _check(code, stops, per_wave, nks)
            if r:
                bad.append((name, 64 * nks, r))
    assert not bad, f"{len(bad)} of them, the first: {bad[:3]}"
