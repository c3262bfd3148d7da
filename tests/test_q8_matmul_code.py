"""What the 8-bit product's compiled kernels have to hold to and the compiler does not see to (no GPU).

Copies from memory to LDS are statements of their own, into which the compiler puts no waits.  Such a
copy takes its LDS address from m0, with one instruction at least between a scalar write of m0 and the
copy, and its descriptor from scalar registers, five after a vector instruction that wrote one.

No vector register goes to scratch memory: one that is loaded again where a branch has switched lanes off
leaves those lanes with a wild value, and such loads stand in the counter that the copies' waits use."""
import os
import re
import subprocess

import pytest

from paper_2406_20037_amd import build


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """(assembly, remarks) of the file as the library has it."""
    out = tmp_path_factory.mktemp("q8") / "s"
    log = subprocess.run(
        [build._hipcc(), *build.HIP_FLAGS, "-Rpass-analysis=kernel-resource-usage", "--cuda-device-only", "-S",
         os.path.join(build.CSRC, "kern_q8_matmul.hip"), "-o", str(out)],
        capture_output=True, text=True, check=True).stderr
    return out.read_text(), log


def scalars(word):
    """The scalar registers that an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)|(m0)", word)
    if not m:
        return set()
    if m[4]:
        return {"m0"}
    return set(range(int(m[1]), int(m[2]) + 1)) if m[1] else {int(m[3])}


def functions(text):
    """Lists of (is a label, words of the line), one a kernel."""
    code = None
    for line in text.splitlines():
        line = line.split(";")[0].strip()
        if re.match(r"_Z\w+:", line):
            code = []
        elif line.startswith(".Lfunc_end"):
            yield code
            code = None
        elif code is not None and re.match(r"\.LBB\w+:", line):
            code.append((True, [line[:-1]]))
        elif code is not None and re.match(r"[a-z]", line):
            code.append((False, line.replace(",", " ").split()))


def early_copies(code):
    """(number of copies, those that something before them comes too close to)."""
    at = {w[0]: i for i, (label, w) in enumerate(code) if label}
    before = {}
    for i, (label, w) in enumerate(code):
        if label or w[0] not in ("s_endpgm", "s_branch"):
            before.setdefault(i + 1, []).append(i)
        if not label and w[0].startswith(("s_branch", "s_cbranch")):
            before.setdefault(at[w[1]], []).append(i)
    copies, early = 0, []
    for i, (label, w) in enumerate(code):
        if label or not w[0].startswith("buffer_load") or "lds" not in w:
            continue
        copies += 1
        held = next(scalars(x) for x in w if x.startswith("s["))
        todo, seen = [(j, 0) for j in before.get(i, [])], set()
        while todo:                                    # backwards over every path, up to five instructions
            j, n = todo.pop()
            if (j, n) in seen or n >= 5:
                continue
            seen.add((j, n))
            if not code[j][0]:
                op, to = code[j][1][0], scalars(code[j][1][1]) if len(code[j][1]) > 1 else set()
                if (n < 1 and "m0" in to) or (op.startswith("v_") and to & held):
                    early.append((code[j][1], w))
                n += int(code[j][1][1], 0) + 1 if op == "s_nop" else 1
            todo += [(k, n) for k in before.get(j, [])]
    return copies, early


def test_the_reader_of_code():
    text = """_Zk:
	v_readfirstlane_b32 s5, v1
	s_mov_b32 m0, s9
.LBB0_1:
	buffer_load_dword v2, s[4:7], 0 offen lds
	s_mov_b32 m0, s9
	s_nop 0
	buffer_load_dwordx4 v2, s[8:11], 0 offen lds
	s_cbranch_scc1 .LBB0_1
.Lfunc_end0:
"""
    (code,) = functions(text)
    copies, early = early_copies(code)
    assert copies == 2 and [e[0][0] for e in early] == ["s_mov_b32", "v_readfirstlane_b32"]


def test_copies_wait_for_their_scalars(compiled):
    total = 0
    for code in functions(compiled[0]):
        copies, early = early_copies(code)
        total += copies
        assert not early, early[:3]
    assert total > 0


def test_no_kernel_spills(compiled):
    names = re.findall(r"Function Name: (\S+)", compiled[1])
    scratch = re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", compiled[1])
    assert len(names) == len(scratch) >= 45
    assert not {n: s for n, s in zip(names, scratch) if s != "0"}


def test_nothing_else_is_warned_of(compiled):
    assert not [x for x in compiled[1].splitlines() if " warning: " in x and "packed-fp32-ops" not in x
                and "--hip-link" not in x]
