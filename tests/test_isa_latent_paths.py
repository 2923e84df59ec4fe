"""The absorbed latent attention's bare products (inline asm, which the compiler does not know as MFMAs), along every path from
each: nothing but the next product that accumulates in place touches a sum in the 18 wait states after it.  (The compiler's own
wait after this instruction is 8.)  Taken branches count: a sum is read behind its loop's exit."""

import os
import re
import shutil
import subprocess

import pytest

from paper_2607_20507_amd import build as B
from tests.test_isa_bare_mfma import _operands

PATTERN = "attn_latent_bf16"


def _tokens(text):
    p = text.split(None, 1)
    return [t.strip().split(" ")[0] for t in p[1].split(",")] if len(p) == 2 else []


def early_uses(lines, pattern, need=18):
    """{kernel: [(bare MFMA, instruction that touches its sum too early, wait states between)]}."""
    out, i = {}, 0
    while i < len(lines):
        m = re.match(r"^(_Z\S*" + pattern + r"\S*):", lines[i])
        i += 1
        if not m:
            continue
        ins, labels, asm = [], {}, False
        while i < len(lines) and not lines[i].startswith(".Lfunc_end"):
            text = lines[i].strip()
            i += 1
            label = re.match(r"(\.LBB\S+):", text)
            if "#ASMSTART" in text or "#ASMEND" in text:
                asm = "#ASMSTART" in text
            elif label:
                labels[label.group(1)] = len(ins)
            elif text and text[0] not in ";.":
                ins.append((text.split(";")[0].strip(), asm))
        out[m.group(1)] = [u for k, (text, bare) in enumerate(ins) if bare and text.startswith("v_mfma") for u in _paths(ins, labels, k, need)]
    return out


def _paths(ins, labels, first, need):
    product = ins[first][0]
    res, found, reached, ahead = _operands(_tokens(product)[0]), [], {}, [(first + 1, 0)]
    while ahead:
        k, states = ahead.pop()
        while k < len(ins) and states < need and reached.get(k, need) > states:
            reached[k] = states
            text = ins[k][0]
            name, ops = text.split()[0], _tokens(text)
            k += 1
            if name == "s_endpgm":
                break
            if name == "s_nop":
                states += int(ops[0]) + 1
                continue
            if name == "s_branch":
                k = labels[ops[0]]
            elif name.startswith("s_cbranch"):
                ahead.append((labels[ops[0]], states + 1))
            elif name.startswith("v_mfma"):
                dst = _operands(ops[0])
                if (_operands(ops[1]) | _operands(ops[2])) & res or (dst & res and dst != res):
                    found.append((product, text, states))
                if dst & res:
                    break  # that product's own uses count from it
            elif not name.startswith("s_") and set().union(*[_operands(t) for t in ops]) & res:
                found.append((product, text, states))
                break
            states += 1
    return found


def test_checker_follows_branches():
    mfma = [";;#ASMSTART", "v_mfma_f32_16x16x32_bf16 a[0:3], v[12:15], v[16:19], a[0:3]", ";;#ASMEND"]
    wait = [";;#ASMSTART", "s_nop 15", "s_nop 7", ";;#ASMEND"]
    read = ["v_accvgpr_read_b32 v8, a3"]

    def count(body):
        return len(early_uses(["_Zattn_latent_bf16_x:"] + body + ["s_endpgm", ".Lfunc_end0:"], PATTERN)["_Zattn_latent_bf16_x"])

    loop = [".LBB0_1:"] + mfma + ["s_cbranch_scc1 .LBB0_3", "s_branch .LBB0_1", ".LBB0_3:"]
    assert count(loop + wait + read) == 0
    assert count(loop + read + wait) == 1  # read before the wait, behind a taken branch
    assert count(loop + ["scratch_store_dwordx4 off, a[0:3], off"] + wait) == 1
    assert count(loop + ["v_mov_b32_e32 v9, v8"] * 18 + read) == 0  # as long by other instructions
    assert count([".LBB0_1:"] + read + mfma + ["s_branch .LBB0_1"]) == 1  # around the loop
    assert count(mfma + mfma + wait + read) == 0


# the GEMMs' bare products: those of gemm_mfma4 wait 18 states, the others pass their sums on to compiler-made products,
# whose copies are to keep the 8
@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="hipcc not available")
@pytest.mark.parametrize("source, checks", [("latent.hip", [(PATTERN, 18, 12)]),
                                            ("gemm.hip", [("gemm_mfma4", 18, 1), ("gemm_mfma2", 8, 1), ("gemm_mfma3", 8, 1)])])
def test_sums_are_read_behind_their_wait(tmp_path, source, checks):
    out = tmp_path / "kernels.s"
    r = subprocess.run([B.hipcc()] + B.flags() + ["--cuda-device-only", "-S", os.path.join(B.CSRC, source), "-o", str(out)],
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = out.read_text().split("\n")
    for pattern, need, kernels in checks:
        uses = early_uses(lines, pattern, need)
        assert len(uses) >= kernels
        for name, found in uses.items():
            assert not found, (name, found[:5])
