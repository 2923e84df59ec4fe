"""CPU checks of the latent attention's planner (host C++): on seeded random batches every
query vector meets every key it sees exactly once, in items within their tiles, and every
part is joined once."""

import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(ROOT, "paper_2607_20507_amd", "csrc")
MAX_PARTS = 512


@pytest.fixture(scope="module")
def plan_exe(tmp_path_factory):
    hipcc = shutil.which("hipcc") or ("/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else None)
    if not hipcc:
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("plan_latent") / "plan_latent_driver")
    subprocess.run([hipcc, "-O1", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", "-I", CSRC, "-I",
                    os.path.join(ROOT, "include"), os.path.join(HERE, "native", "plan_latent_driver.cpp"),
                    os.path.join(CSRC, "latent_plan.cpp"), "-o", exe], check=True, capture_output=True)
    return exe


def segments(rng, n, rows, keys):
    segs, r0, page, skip = [], 0, 0, 0
    for _ in range(n):
        r, p = int(rng.integers(1, rows + 1)), int(rng.integers(0, keys + 1))
        segs.append((r0, r, p, page, skip))
        r0, page = r0 + r, page + (r + p + 15) // 16
        skip += int(rng.integers(0, 3))  # rows of the other form in between
    return segs


def run(exe, problems):
    text = []
    for H, waves, segs in problems:
        text.append(f"{H} {waves} {len(segs)}")
        text += [" ".join(map(str, s)) for s in segs]
    out = subprocess.run([exe], input="\n".join(text) + "\n", capture_output=True, text=True, check=True).stdout
    plans = []
    for line in out.splitlines():
        f = line.split()
        v = tuple(int(x) for x in f[1:])
        if f[0] == "plan":
            plans.append({"plan": v, "item": [], "group": [], "block": [], "join": []})
        elif f[0] == "prompt":
            plans[-1]["prompt"] = v
        else:
            plans[-1][f[0]].append(v)
    assert len(plans) == len(problems)
    return plans


def check(items, groups, n_parts, tile, step, segs, unit, rows_of, prompt):
    """unit: query vectors a row; rows_of(segment): its first row in the items' numbers."""
    cover, parts = {}, {}
    for qv0, nqv, row0, pos0, page0, t0, t1, part, qoff in items:
        seg = next(s for s in segs if rows_of(s) * unit <= qv0 < (rows_of(s) + s[1]) * unit)
        assert 1 <= nqv <= tile and qv0 + nqv <= (rows_of(seg) + seg[1]) * unit and page0 == seg[3]
        assert t0 % step == 0 and 0 <= t0 < t1
        last = seg[2] + (qv0 + nqv - 1) // unit - rows_of(seg)  # its last row's position
        assert t1 <= last + 1
        if prompt:
            assert pos0 == seg[2] + qv0 - rows_of(seg)
        else:
            assert row0 == seg[0] and pos0 == seg[2] and qoff == seg[4]
        cover.setdefault((qv0, nqv, last), []).append((t0, t1))
        if part >= 0:
            assert part not in parts
            parts[part] = (qv0, nqv, t0)
    for (_, _, last), ranges in cover.items():
        ranges.sort()
        assert ranges[0][0] == 0 and ranges[-1][1] == last + 1
        assert all(a[1] == b[0] for a, b in zip(ranges, ranges[1:]))
    vectors = sorted((q, n) for q, n, _ in cover)
    assert all(a[0] + a[1] <= b[0] for a, b in zip(vectors, vectors[1:]))
    assert sum(n for _, n in vectors) == unit * sum(s[1] for s in segs)
    assert sorted(parts) == list(range(n_parts)) and n_parts <= MAX_PARTS
    joined = 0
    for qv0, nqv, part0, nparts in groups:
        mine = [parts[part0 + i] for i in range(nparts)]
        assert nparts >= 2 and all(m[:2] == (qv0, nqv) for m in mine) and len({m[2] for m in mine}) == nparts
        joined += nparts
    assert joined == n_parts
    lengths = [i[6] - i[5] for i in items]
    assert lengths == sorted(lengths, reverse=True)


def test_random_batches(plan_exe):
    rng = np.random.default_rng(7)
    problems = []
    for _ in range(150):
        H = int(rng.choice([1, 3, 8, 11, 16, 32, 40, 128, 300]))
        n, rows, keys = [(1, 8, 9000), (1, 2000, 3000), (64, 8, 4096), (5, 40, 600), (200, 1, 300), (3, 1, 200000)][int(rng.integers(6))]
        problems.append((H, int(rng.choice([0, 0, 4, 8])), segments(rng, n, rows, keys)))
    for (H, waves, segs), p in zip(problems, run(plan_exe, problems)):
        tile, n_parts = p["plan"]
        assert tile in ((16,) if waves else (16, 32, 64))
        check(p["item"], p["group"], n_parts, tile, 32, segs, H, lambda s: s[0], False)
        rows, n_parts = p["prompt"]
        assert rows in (128, 256)
        check(p["block"], p["join"], n_parts, rows, 64, segs, 1, lambda s: s[0] + s[4], True)


def test_tiles_and_whole_items(plan_exe):
    """Tiles by a sequence's query vectors; contexts whole up to four chunks a wave; one item a CU otherwise."""
    def plan(H, rows, pos0, waves=0):
        return run(plan_exe, [(H, waves, [(0, rows, pos0, 0, 0)])])[0]
    assert [plan(h, 1, 100)["plan"][0] for h in (1, 16, 17, 32, 33, 64, 65, 128)] == [16, 16, 32, 32, 64, 64, 64, 64]
    assert plan(32, 1, 100, 8)["plan"][0] == 16
    assert plan(16, 1, 511)["plan"][1] == 0 and plan(16, 1, 512)["plan"][1] > 0
    assert plan(32, 1, 255)["plan"][1] == 0 and plan(32, 1, 256)["plan"][1] > 0
    assert plan(64, 1, 127)["plan"][1] == 0 and plan(64, 1, 128)["plan"][1] > 0
    assert plan(16, 1, 255, 8)["plan"][1] == 0 and plan(16, 1, 256, 8)["plan"][1] > 0
    assert len(plan(16, 1, (1 << 20) - 1)["item"]) == 256
