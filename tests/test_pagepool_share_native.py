"""CPU checks of pages that several tables hold (csrc/pages.h): a random script
against a plain model, in which a page is free exactly when no table holds it,
the lowest-numbered free page is taken first and compaction moves the held pages
from the end to the free ones at the front, both in ascending order."""

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
    out = str(tmp_path_factory.mktemp("pps") / "pagepool_share_driver")
    subprocess.run([gxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2607_20507_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "pagepool_share_driver.cpp"), "-o", out], check=True)
    return out


@pytest.mark.parametrize("seed", range(4))
def test_sharing_and_compaction(exe, seed):
    rng = np.random.default_rng(seed)
    num = 50
    tabs, script, want = {}, [], []

    def held():
        return {p for t in tabs.values() for p in t}

    for _ in range(500):
        op = rng.choice(["E", "E", "T", "F", "K"])
        a = int(rng.integers(0, 8))
        t = tabs.get(a, [])
        if op == "E":
            n = 16 * len(t) + int(rng.integers(0, 60))
            script.append(f"E {a} {n}")
            more = (n + 15) // 16 - len(t)
            free = sorted(set(range(num)) - held())
            if more > len(free):
                head = "oom"
                tabs.setdefault(a, [])
            else:
                head = "ok"
                tabs[a] = t + free[:max(0, more)]
        elif op == "T":
            n = int(rng.integers(0, 16 * len(t) + 1))
            script.append(f"T {a} {n}")
            tabs[a] = t[:(n + 15) // 16]
            head = "ok"
        elif op == "F":
            b = 100 + len(script)
            script.append(f"F {a} {b}")
            tabs.setdefault(a, [])
            tabs[b] = list(t)
            head = "ok"
            if len(tabs) > 14:  # keep the script's tables few
                want.append((head, {k: list(v) for k, v in tabs.items()}))
                gone = sorted(k for k in tabs if k >= 100)[0]
                script.append(f"T {gone} 0")
                tabs[gone] = []
        else:
            script.append("K 0 0")
            live = len(held())
            moves = list(zip(sorted(p for p in held() if p >= live), sorted(set(range(live)) - held())))
            name = dict(moves)
            tabs = {k: [name.get(p, p) for p in v] for k, v in tabs.items()}
            head = " ".join(["moved"] + [f"{x}>{y}" for x, y in moves])
            assert held() == set(range(live))
        want.append((head, {k: list(v) for k, v in tabs.items()}))
    out = subprocess.run([exe], input=f"{num}\n" + "\n".join(script) + "\n", capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(want)
    for line, (head, tables) in zip(out, want):
        first, *parts = line.split(" |")
        everything = [p for t in tables.values() for p in t]
        assert first == f"{head} free {num - len(set(everything))}"
        got = {int(p.split(":")[0]): p.split(":")[1].split() for p in parts}
        for k, t in tables.items():
            assert got.get(k, []) == [f"{p}*" if everything.count(p) > 1 else str(p) for p in t]
