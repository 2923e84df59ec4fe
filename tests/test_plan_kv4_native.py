"""CPU checks of the planner of the attention over a 4-bit cache (plan_kv4, host
C++): the invariants of its items on seeded random batches, and its rules for
tiles, waves and splits at their borders."""

import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(ROOT, "paper_2607_20507_amd", "csrc")


@pytest.fixture(scope="module")
def plan_exe(tmp_path_factory):
    hipcc = shutil.which("hipcc") or ("/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else None)
    if not hipcc:
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("plan_kv4") / "plan_kv4_driver")
    subprocess.run([hipcc, "-O1", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", "-I", CSRC, "-I",
                    os.path.join(ROOT, "include"), os.path.join(HERE, "native", "plan_kv4_driver.cpp"),
                    os.path.join(CSRC, "plan.cpp"), "-o", exe], check=True, capture_output=True)
    return exe


def run_plans(exe, problems):
    text = []
    for G, Hkv, max_parts, fp32, segs in problems:
        text.append(f"{G} {Hkv} {max_parts} {int(fp32)} {len(segs)}")
        text += [f"{s} {r0} {n} {p0}" for s, r0, n, p0 in segs]
    out = subprocess.run([exe], input="\n".join(text) + "\n", capture_output=True, text=True, check=True).stdout
    plans = []
    for line in out.splitlines():
        f = line.split()
        if f[0] == "plan":
            plans.append({"nt": int(f[1]), "w": int(f[2]), "prefill": bool(int(f[3])), "n_parts": int(f[4]), "items": [], "groups": []})
        else:
            plans[-1][f[0] + "s"].append(tuple(int(x) for x in f[1:]))
    assert len(plans) == len(problems)
    return plans


def segments(rng, n, rows, keys):
    segs, r0 = [], 0
    for i in range(n):
        r = int(rng.integers(1, rows + 1))
        segs.append((i, r0, r, int(rng.integers(0, keys + 1))))
        r0 += r
    return segs


def check(plan, G, Hkv, max_parts, fp32, segs):
    by_seq = {s: (r0, n, p0) for s, r0, n, p0 in segs}
    cover, parts = {}, {}
    for row0, nrows, pos0, seq, t0, t1, part in plan["items"]:
        r0, n, p0 = by_seq[seq]
        assert nrows >= 1 and r0 <= row0 and row0 + nrows <= r0 + n and pos0 == p0 + row0 - r0
        assert 0 <= t0 < t1 <= pos0 + nrows
        assert plan["prefill"] or nrows * G <= 16 * plan["nt"]
        if part >= 0:
            assert part not in parts
            parts[part] = (row0, nrows)
        for r in range(row0, row0 + nrows):
            cover.setdefault(r, []).append((t0, t1))
    for s, r0, n, p0 in segs:
        for r in range(r0, r0 + n):
            ranges = sorted(cover.pop(r))
            assert ranges[0][0] == 0 and ranges[-1][1] >= p0 + r - r0 + 1  # the row's last key
            assert all(a[1] == b[0] for a, b in zip(ranges, ranges[1:]))
    assert not cover and len(parts) == plan["n_parts"] <= max_parts
    for row0, nrows, part0, nparts in plan["groups"]:
        assert nparts >= 2
        for p in range(part0, part0 + nparts):
            assert parts.pop(p) == (row0, nrows)
    assert not parts
    if plan["prefill"]:
        assert not fp32 and min(n for _, _, n, _ in segs) >= 64 and 256 % G == 0
        assert max(n + p for _, _, n, p in segs) <= 16384
    else:
        assert plan["w"] in (4, 8) and plan["nt"] in ((1, 2) if fp32 else (1, 2, 4))
        assert plan["w"] == 4 or (plan["nt"] < 4 and not fp32)


def test_plans_cover_every_row_and_key_once(plan_exe):
    rng = np.random.default_rng(8)
    problems = []
    for i in range(300):
        fp32 = bool(rng.integers(0, 2))
        G = int(rng.choice([1, 2, 3, 4, 7, 8, 16, 32] + ([] if fp32 else [48, 64])))
        n = int(rng.integers(1, 40))
        rows = int(rng.choice([1, 4, 8, 70, 200]))
        keys = int(rng.choice([0, 15, 500, 3000, 20000]))
        problems.append((G, int(rng.choice([1, 2, 8, 16])), int(rng.choice([4096, 64, 3])), fp32, segments(rng, n, rows, keys)))
    problems.append((4, 8, 4096, False, [(0, 0, 1, 2 ** 31 - 17)]))  # the longest cache
    for plan, problem in zip(run_plans(plan_exe, problems), problems):
        check(plan, *problem)


def test_rules(plan_exe):
    one = lambda rows, keys: [(0, 0, rows, keys)]  # noqa: E731
    many = lambda n, rows, keys: [(i, i * rows, rows, keys) for i in range(n)]  # noqa: E731
    problems = [
        (4, 8, 4096, False, one(6, 2047)),         # a short single sequence: whole, eight waves
        (4, 8, 4096, False, one(1, 131000)),       # a long one: 64 parts a kv head
        (4, 8, 4096, False, many(64, 8, 992)),     # 512 workgroups: four waves, whole
        (16, 8, 4096, False, many(8, 4, 2000)),    # the widest tiles: split for 256 workgroups
        (4, 8, 4096, False, many(2, 64, 0)),       # prompts
        (4, 8, 4096, True, many(2, 64, 0)),        # fp32 prompts keep the tiled form
        (7, 1, 4096, False, one(64, 0)),           # so do groups that do not divide a block
        (4, 8, 4096, False, one(64, 16400)),       # and contexts beyond the prompt kernel's page list
    ]
    p = run_plans(plan_exe, problems)
    assert (p[0]["nt"], p[0]["w"], p[0]["n_parts"]) == (1, 8, 0)
    assert (p[1]["nt"], p[1]["w"], p[1]["n_parts"]) == (1, 4, 64)
    assert (p[2]["nt"], p[2]["w"], p[2]["n_parts"]) == (2, 4, 0)
    assert (p[3]["nt"], p[3]["w"]) == (4, 4) and len(p[3]["items"]) == 32
    assert p[4]["prefill"] and not p[5]["prefill"] and not p[6]["prefill"] and not p[7]["prefill"]
