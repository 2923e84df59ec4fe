"""CPU checks of the 4-bit cache's byte order and scales (csrc/kv4_layout.h)
against the float64 definition."""

import os
import shutil
import subprocess

import numpy as np
import pytest

import kv4_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("kv4") / "kv4_layout_driver")
    subprocess.run([gxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2607_20507_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "kv4_layout_driver.cpp"), "-o", exe], check=True)
    return exe


def test_layout_is_a_bijection_inside_the_block(driver):
    lines = subprocess.run([driver], input="", capture_output=True, text=True, check=True).stdout.split("\n")
    rows = np.array([[int(x) for x in line.split()] for line in lines if line])
    for hd in (64, 128):
        of = rows[rows[:, 0] == hd]
        for place, (byte, nib, scale) in ((ref.k_place, (3, 4, 5)), (ref.v_place, (6, 7, 8))):
            for row in of:
                assert place(row[1], row[2], hd) == (row[byte], row[nib], row[scale])
            where = of[:, byte] * 2 + of[:, nib]
            assert sorted(where) == list(range(16 * hd))  # every nibble of the codes once
            assert of[:, scale].min() == 8 * hd and of[:, scale].max() == ref.block_bytes(hd) - 1
            # a scale byte per (token, block of 32), tokens never share a byte
            assert len({(r[1], r[2] // 32) for r in of}) == len(set(of[:, scale])) == 16 * hd // 32
            assert len({(r[1], r[byte]) for r in of}) == len(set(of[:, byte]))


def test_scales_match_the_definition(driver):
    rng = np.random.default_rng(3)
    x = np.concatenate([np.float32(2.0) ** rng.uniform(-149, 127, 2000), [0.0, 6.0, np.nextafter(np.float32(6), np.float32(9)), 1.5, 0.75, 3.4e38],
                        [1e-45, 2.0 ** -126, 6 * 2.0 ** -126, np.inf]]).astype(np.float32)
    out = subprocess.run([driver], input="\n".join(str(b) for b in x.view(np.uint32)), capture_output=True, text=True,
                         check=True).stdout.split("\n")
    got = [int(v) for v in out if v and " " not in v]
    assert len(got) == len(x)
    for v, s in zip(x.astype(np.float64), got):
        block = np.zeros(32)
        block[7] = v
        assert s == ref.quantise(block)[1][0], v


def test_reference_rounds_ties_to_even_codes():
    x = np.zeros(32)
    x[:9] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.75]
    np.testing.assert_array_equal(ref.held(x)[:9], [6, 0, 1, 1, 2, 2, 4, 4, -1])
