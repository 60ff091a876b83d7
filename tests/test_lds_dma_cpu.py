"""The wait states before LDS DMA in the built kernels, which inline asm has to hold itself: read from the library's own code."""
import os
import re
import subprocess

import pytest

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def registers(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)", operand)
    return set() if m is None else {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))


def states(op, args):
    return 1 + int(args[0], 0) if op == "s_nop" else 1


def faults(listing):
    """(number of LDS DMA loads, those that come too early), of llvm-objdump's lines."""
    n, early, before, name = 0, [], [], None
    for line in listing:
        head = re.match(r"[0-9a-f]+ <(\S+)>:", line)
        if head:
            name, before = head[1], []
        m = re.match(r"\s+([a-z]\w*)\s*(.*?)\s*//", line)
        if head or not m:
            continue
        op, args = m[1], m[2].replace(",", " ").split()
        if op.startswith("global_load_lds"):
            n += 1
            base = set().union(*map(registers, args))
            waited = 0
            for o, a in reversed(before):
                # a write of M0 needs one wait state, a vector instruction's write of the base five
                if a and (a[0] == "m0" and waited < 1 or o.startswith("v_") and registers(a[0]) & base):
                    early.append((name, o, a, op, args))
                waited += states(o, a)
                if waited >= 5 or a and not o.startswith("v_") and registers(a[0]) & base:
                    break
        before = before[-8:] + [(op, args)]
    return n, early


def listing(*lines):
    return ["0000 <kernel>:"] + [f"\t{x}   // 000: 00" for x in lines]


def test_what_comes_too_early():
    load = "global_load_lds_dwordx4 v1, s[4:5]"
    assert faults(listing("s_mov_b32 m0, s2", load))[1] and not faults(listing("s_mov_b32 m0, s2", "s_nop 0", load))[1]
    assert faults(listing("v_readfirstlane_b32 s5, v3", "s_mov_b32 m0, s2", "s_nop 2", load))[1]
    assert not faults(listing("v_readfirstlane_b32 s5, v3", "s_mov_b32 m0, s2", "s_nop 3", load))[1]
    assert not faults(listing("v_readfirstlane_b32 s7, v3", "s_mov_b32 m0, s2", "s_mov_b64 s[4:5], s[6:7]", load))[1]
    assert faults(listing(load, load)) == (2, [])


@pytest.mark.parametrize("library", ["OUT", "CALIB_OUT"])
def test_lds_dma_waits(library, tmp_path):
    from paper_2609_29029_amd import build as B
    if not os.path.exists(OBJDUMP):
        pytest.skip("no ROCm llvm-objdump in this image")
    path = getattr(B, library)
    if not os.path.exists(path):
        B.build()
    os.symlink(path, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    total = 0
    for name in sorted(os.listdir(tmp_path)):
        if name.endswith(B.ARCH):
            text = subprocess.run([OBJDUMP, "-d", name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
            n, early = faults(text.splitlines())
            total += n
            assert not early, (len(early), early[0])
    assert total > 0
