"""The absorbed latent attention issues its MFMAs as bare inline asm, which the compiler
does not know as MFMAs.  Checked on the compiled kernels: no vector instruction writes an
operand of one in the two wait states before it, and none touches a result in the 18 after
it, but for the next product that accumulates in place."""

import os
import re
import shutil
import subprocess

import pytest

from paper_2607_20507_amd import build as B
from tests.test_isa_bare_mfma import _operands, unwaited_writes

PATTERN = "attn_latent_bf16"


def early_uses(lines, pattern, need=18):
    """{kernel: [(bare MFMA, instruction that touches its result too early)]}, along the straight path from each."""
    out, name = {}, None
    for i, l in enumerate(lines):
        m = re.match(r"^(_Z\S*" + pattern + r"\S*):", l)
        if m:
            name = m.group(1)
            out[name] = []
        elif l.startswith(".Lfunc_end"):
            name = None
        if name is None or not l.strip().startswith("v_mfma") or "#ASMSTART" not in lines[i - 1]:
            continue
        res = _operands(l.split(None, 1)[1].split(",")[0].strip())
        states, j = 0, i + 1
        while states < need and j < len(lines) and not lines[j].startswith(".Lfunc_end"):
            p = lines[j].strip().split(None, 1)
            j += 1
            if not p or p[0].startswith((";", ".")) or p[0].endswith(":"):
                continue
            if p[0] == "s_nop":
                states += int(p[1]) + 1
                continue
            if p[0] in ("s_branch", "s_endpgm"):
                break
            if p[0].startswith("v_mfma"):
                ops = [t.strip() for t in p[1].split(",")]
                dst = _operands(ops[0])
                if (_operands(ops[1]) | _operands(ops[2])) & res or (dst & res and dst != res):
                    out[name].append((l.strip(), lines[j - 1].strip()))
                if dst == res:
                    break
            elif len(p) == 2 and not p[0].startswith("s_"):
                if set().union(*[_operands(t.strip().split(" ")[0]) for t in p[1].split(",")]) & res:
                    out[name].append((l.strip(), lines[j - 1].strip()))
            states += 1
    return out


def test_checker_flags_an_early_use():
    mfma = [";;#ASMSTART", "v_mfma_f32_16x16x32_bf16 v[0:3], v[12:15], v[16:19], v[0:3]", ";;#ASMEND"]
    k = ["_Zattn_latent_bf16_x:"] + mfma
    assert early_uses(k + ["s_nop 15", "s_nop 7", "v_mov_b32_e32 v8, v3"], PATTERN)["_Zattn_latent_bf16_x"] == []
    assert len(early_uses(k + ["s_nop 15", "v_mov_b32_e32 v8, v3"], PATTERN)["_Zattn_latent_bf16_x"]) == 1
    assert early_uses(k + mfma, PATTERN)["_Zattn_latent_bf16_x"] == []
    assert len(early_uses(k + ["v_mfma_f32_16x16x32_bf16 v[4:7], v[0:3], v[16:19], v[4:7]"], PATTERN)["_Zattn_latent_bf16_x"]) == 1


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="hipcc not available")
def test_latent_products(tmp_path):
    out = tmp_path / "latent.s"
    cmd = [B.hipcc()] + B.flags() + ["--cuda-device-only", "-S", os.path.join(B.CSRC, "latent.hip"), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = out.read_text().split("\n")
    writes, uses = unwaited_writes(lines, PATTERN), early_uses(lines, PATTERN)
    assert len(writes) == 12 and writes.keys() == uses.keys()
    for name, (n, bad) in writes.items():
        assert n >= 32 and not bad, (name, n, bad[:5])
        assert not uses[name], (name, uses[name][:5])
