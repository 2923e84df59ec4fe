"""CPU checks of a table cut to a length (csrc/pages.h, what a rollback does to
the pages): the slots to clear are every position from the new length on, but
for those in pages that another table holds; a page held by others that the new
length ends in is replaced by a copy, whose slots from the length on are cleared
too.  At lengths that end a page and at others, against a plain model."""

import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("g++ not available")
    out = str(tmp_path_factory.mktemp("ppc") / "pagepool_cut_driver")
    subprocess.run([gxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2607_20507_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "pagepool_cut_driver.cpp"), "-o", out], check=True)
    return out


def run(exe, num, script):
    out = subprocess.run([exe], input=f"{num}\n" + "\n".join(script) + "\n", capture_output=True, text=True, check=True).stdout
    got = []
    for line in out.splitlines():
        head, *tables = line.split(" |")
        words = head.split()
        got.append((words[:words.index("free")], int(words[-1]),
                    {int(t.split(":")[0]): [int(p.rstrip("*")) for p in t.split(":")[1].split()] for t in tables}))
    return got


@pytest.mark.parametrize("keep, count", [(0, 40), (15, 25), (16, 24), (17, 23), (32, 8), (39, 1), (40, 0)])
def test_every_position_from_the_new_length_on(exe, keep, count):
    got = run(exe, 8, ["E 1 40", f"C 1 {keep} 40"])
    assert got[1][0][:2] == ["cut", "-1>-1"]
    assert sorted(map(int, got[1][0][2:])) == list(range(keep, 40)) and len(got[1][0]) - 2 == count


@pytest.mark.parametrize("seed", range(6))
def test_against_a_model(exe, seed):
    rng = np.random.default_rng(seed)
    num, tabs, ends, script, want = 40, {}, {}, [], []
    for step in range(400):
        held = {p for t in tabs.values() for p in t}
        free = sorted(set(range(num)) - held)
        a = int(rng.integers(0, 6))
        t = tabs.setdefault(a, [])
        op = rng.choice(["E", "C", "C", "F"])
        if op == "E":
            n = 16 * len(t) + int(rng.integers(0, 50))
            script.append(f"E {a} {n}")
            more = (n + 15) // 16 - len(t)
            if more > len(free):
                want.append(["oom"])
            else:
                tabs[a], ends[a] = t + free[:max(0, more)], n
                want.append(["ok"])
        elif op == "F":
            b = 100 + step
            script.append(f"F {a} {b}")
            tabs[b], ends[b] = list(t), 16 * len(t)
            want.append(["ok"])
        else:
            if rng.random() < 0.5 and len(tabs) > 6:
                a = sorted(tabs)[-1]
                t = tabs[a]
            end = int(rng.integers(max(0, 16 * len(t) - 20), 16 * len(t) + 1))
            keep = int(rng.choice([0, rng.integers(0, end + 1), end // 16 * 16, min(end, 16)]))
            script.append(f"C {a} {keep} {end}")
            others = {p for k, v in tabs.items() if k != a for p in v}
            gone = [p for p in t[(keep + 15) // 16:] if p not in others]
            copied = keep % 16 != 0 and t[keep // 16] in others
            if copied and not free and not gone:
                want.append(["oom"])
            else:
                clear = {t[p // 16] * 16 + p % 16 for p in range(keep, end) if t[p // 16] not in others}
                tabs[a] = t[:(keep + 15) // 16]
                frm = to = -1
                if copied:
                    frm, to = t[keep // 16], min(free + gone)
                    clear = {s for s in clear if s // 16 != to}
                    clear |= {to * 16 + p % 16 for p in range(keep, min(end, keep // 16 * 16 + 16))}
                    tabs[a][-1] = to
                want.append(["cut", f"{frm}>{to}", clear])
        want[-1] = (want[-1], {k: list(v) for k, v in tabs.items()})
    got = run(exe, num, script)
    assert len(got) == len(want)
    for line, ((head, _, tables), (w, wt)) in enumerate(zip(got, want)):
        assert head[:2] == w[:2], script[line]
        if w[0] == "cut":
            slots = [int(s) for s in head[2:]]
            assert len(slots) == len(set(slots)) and set(slots) == w[2], script[line]
        assert {k: v for k, v in tables.items() if v} == {k: v for k, v in wt.items() if v}, script[line]


def test_giving_up_pages_allocates_nothing(exe):
    """Also after a compaction: the calls that give up pages pass no exception on."""
    script = [f"E {i} 64" for i in range(10)] + ["C 3 0 64", "C 7 16 64", "K 0 0", "D 0 0", "E 1 640", "D 0 0"]
    got = run(exe, 40, script)
    assert [g[0] for g in got if g[0][0] == "allocated"] == [["allocated", "0"]] * 2
