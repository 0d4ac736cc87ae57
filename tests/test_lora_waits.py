"""The copies of activations into LDS that lora_gemm.hip keeps under way (CPU: the kernels are compiled to gfx950
assembly and every path through them is followed; nothing runs on a GPU).

A step multiplies a slot that a load to LDS filled steps before.  Such a load has no destination register, so the
compiler waits for none: the step's own s_waitcnt has to leave at most the copies of the ST - 2 steps behind it under
way, counted in the instructions that are really there (the compiler drops loads of codes that no later step uses)."""
import os
import re
import shutil
import subprocess

import pytest

from qmlp_testutil import CSRC

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")

# lora_gemm_kernel<bits, BM, BN, WM, WN, ST, split>: ST slots, BM / (8 waves) copies of a wave and step;
# lora_mid_kernel<bits, WM>: four slots, WM copies
GEMM = re.compile(r"lora_gemm_kernelILi(\d)ELi(\d+)ELi(\d+)ELi(\d)ELi(\d)ELi(\d)ELb([01])E")
MID = re.compile(r"lora_mid_kernelILi(\d)ELi(\d)E")


def copies_and_slots(name):
    m = GEMM.search(name)
    if m:
        bm, bn, wm, wn, st = (int(m.group(i)) for i in range(2, 7))
        waves = bm // (32 * wm) * (bn // (32 * wn))
        return bm // (8 * waves), st
    m = MID.search(name)
    return (int(m.group(2)), 4) if m else None


def instructions(text):
    """{kernel: [(kind, argument)]} of what the vector memory counter and the control flow depend on."""
    out, cur, asm = {}, None, False
    for line in text.splitlines():
        s = line.strip()
        m = re.match(r"^(_Z\S+):", line)
        if m:
            cur = out.setdefault(m.group(1), [])
        if cur is None or not s:
            continue
        if s.startswith(";;#ASMSTART") or s.startswith(";#ASMSTART"):
            asm = True
        elif s.startswith(";;#ASMEND") or s.startswith(";#ASMEND"):
            asm = False
        elif re.match(r"^\.LBB\S+:", s):
            cur.append(("label", s.split(":")[0]))
        elif re.match(r"^(buffer|global|flat|scratch)_(load|store|atomic)", s):
            cur.append(("mem", "x" if re.search(r"\blds\b", s) else "o"))
        elif s.startswith("s_waitcnt") and "vmcnt" in s:
            cur.append(("wait", int(re.search(r"vmcnt\((\d+)\)", s).group(1))))
        elif s.startswith("s_barrier"):
            cur.append(("step" if asm else "barrier", None))       # (the step's barrier is written by hand)
        elif s.startswith("s_cbranch"):
            cur.append(("maybe", s.split()[1]))
        elif s.startswith("s_branch"):
            cur.append(("jump", s.split()[1]))
        elif s.startswith("s_endpgm"):
            cur.append(("end", None))
    return out


def most_under_way(code):
    """The most copies (x) that are under way at a step's barrier, on any path: (count, steps' barriers seen)."""
    at = {a: i for i, (k, a) in enumerate(code) if k == "label"}
    seen, work, worst, steps = set(), [(0, "")], 0, set()
    while work:
        pc, q = work.pop()
        while True:
            if pc >= len(code):
                break
            kind, arg = code[pc]
            if kind == "label":
                if (pc, q) in seen:
                    break
                seen.add((pc, q))
            elif kind == "mem":
                q = (q + arg)[-64:]
            elif kind == "wait":
                q = q[-arg:] if arg else ""
            elif kind == "step":
                worst = max(worst, q.count("x"))
                steps.add(pc)
            elif kind == "maybe":
                work.append((at[arg], q))
            elif kind == "jump":
                pc = at[arg]
                continue
            elif kind == "end":
                assert "x" not in q, "a copy outlives its workgroup"
                break
            pc += 1
    return worst, len(steps)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "lora_gemm.s"
    from paper_2606_04238_amd.build import COMMON
    flags = [f for f in COMMON if f != "-fPIC"]
    subprocess.run([HIPCC] + flags + ["-S", "--cuda-device-only", os.path.join(CSRC, "lora_gemm.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    return {k: v for k, v in instructions(out.read_text()).items() if copies_and_slots(k)}


def test_every_kernel_is_there(kernels):
    assert sum(bool(GEMM.search(k)) for k in kernels) == 6 and sum(bool(MID.search(k)) for k in kernels) == 4


def test_copies_have_arrived(kernels):
    for name, code in sorted(kernels.items()):
        copies, slots = copies_and_slots(name)
        worst, steps = most_under_way(code)
        assert steps > 0, name
        assert worst <= (slots - 2) * copies, "%s: %d copies under way, %d belong to later steps" % (
            name, worst, (slots - 2) * copies)


def test_a_load_that_the_compiler_drops_is_found():
    """A window that counts on two loads of codes a step, in a tail where they are gone."""
    loop = [("label", "a"), ("wait", 8), ("step", None), ("mem", "x"), ("mem", "x"), ("mem", "o"), ("mem", "o"), ("maybe", "a")]
    tail = [("wait", 8), ("step", None), ("mem", "x"), ("mem", "x")] * 2 + [("wait", 8), ("step", None), ("wait", 0), ("end", None)]
    start = [("mem", "x")] * 6 + [("mem", "o")] * 10
    assert most_under_way(start + loop + [("wait", 0), ("end", None)])[0] == 4
    assert most_under_way(start + loop + tail)[0] == 6
