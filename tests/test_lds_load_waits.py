"""The waits that gfx9 wants before a load to LDS written in inline asm.

Two of its rules are kept by instructions put between by hand or by the
compiler: one wait state from a scalar write of M0 to a load to LDS that reads it,
and five from a vector instruction's write of a scalar register to a memory
instruction that takes its address there.  The compiler keeps them for its own
instructions and does not look into asm.  Each source is compiled to assembly
(CPU only) and every load to LDS is followed back over all ways that lead to it."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_33614_amd import build as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.HIPCC) or shutil.which("hipcc") is None, reason="hipcc missing")
SOURCES = ["ce.hip", "balance.hip", "wide.hip"]


def registers(operand):
    m = re.match(r"s\[(\d+):(\d+)\]$", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.match(r"s(\d+)$", operand)
    return {int(m[1])} if m else {"m0"} if operand == "m0" else {"vcc"} if operand == "vcc" else set()


def parse(text):
    """[(opcode, operands)] of every instruction, and a label's place in it."""
    code, labels = [], {}
    for line in text.splitlines():
        line = line.split(";")[0].split("//")[0].strip()
        if re.match(r"[\w.$]+:$", line):
            labels[line[:-1]] = len(code)
        elif line and not line.startswith("."):
            op, _, rest = line.partition(" ")
            code.append((op, [p.split()[0] for p in rest.split(",") if p.strip()]))
    return code, labels


def too_close(code, before, at, states, writes):
    """Whether, on some way to code[at], an instruction for which `writes` holds
    lies fewer than `states` wait states before it."""
    todo, seen = [(at, 0)], {}
    while todo:
        i, passed = todo.pop()
        for j in before[i]:
            op, args = code[j]
            if writes(op, args):
                return True
            now = passed + (1 + int(args[0], 0) if op == "s_nop" else 1)
            if now < states and seen.get(j, states) > now:
                seen[j] = now
                todo.append((j, now))
    return False


def faults(text):
    code, labels = parse(text)
    before = [[] for _ in range(len(code) + 1)]
    for i, (op, args) in enumerate(code):
        if op.startswith(("s_branch", "s_cbranch")) and args and args[0] in labels:
            before[labels[args[0]]].append(i)
        if op not in ("s_branch", "s_endpgm", "s_setpc_b64"):
            before[i + 1].append(i)
    loads, out = 0, []
    for i, (op, args) in enumerate(code):
        if not re.match(r"(global|scratch|buffer)_load.*lds", op) and not (op.startswith("buffer_load") and "lds" in args):
            continue
        loads += 1
        if too_close(code, before, i, 1, lambda o, a: o.startswith("s_") and a[:1] == ["m0"]):
            out.append((i, "M0"))
        address = set().union(*[registers(a) for a in args])
        if address and too_close(code, before, i, 5, lambda o, a: o.startswith("v_") and a and bool(registers(a[0]) & address)):
            out.append((i, "address"))
    return loads, out


@pytest.mark.parametrize("src", SOURCES)
def test_loads_to_lds_keep_their_waits(src, tmp_path):
    out = str(tmp_path / "k.s")
    r = subprocess.run([B.HIPCC, *B.CFLAGS, "--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    loads, bad = faults(open(out).read())
    assert loads > 50 and not bad, (loads, bad[:8])


def test_every_source_with_such_asm_is_looked_at():
    has = {f for f in os.listdir(B.CSRC) if "asm volatile" in (s := open(os.path.join(B.CSRC, f)).read()) and "load_lds" in s}
    assert has == {"wide.hip", "loss_gemm.h"}            # (the header's kernels are in ce.hip and balance.hip)


def test_the_check_sees_a_missing_wait():
    load = "\tglobal_load_lds_dwordx4 v2, s[4:5]\n"
    head, end = "k:\n\tv_readfirstlane_b32 s5, v1\n", "\ts_endpgm\n"
    assert faults(head + "\ts_nop 4\n\ts_mov_b32 m0, s8\n\ts_nop 0\n" + load + end) == (1, [])
    assert faults(head + "\ts_nop 4\n\ts_mov_b32 m0, s8\n" + load + end)[1] == [(3, "M0")]
    assert faults(head + "\ts_nop 1\n\ts_mov_b32 m0, s8\n\ts_nop 0\n" + load + end)[1] == [(4, "address")]
    # over the back edge of a loop
    loop = "k:\n.L1:\n\ts_add_i32 m0, s8, 64\n\ts_nop 0\n" + load + "\tv_readfirstlane_b32 s4, v1\n\ts_cbranch_scc1 .L1\n" + end
    assert faults(loop)[1] == [(2, "address")]
