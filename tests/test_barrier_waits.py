"""At every barrier of every built kernel a wave's LDS writes have been waited for: a walk over the kernels' instructions as the
library holds them (host only). What another wave reads behind a barrier is otherwise whatever stood there before, now and then."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2602_04361_amd import build as B
from paper_2602_04361_amd import sparvar as sv
from test_kernel_registers import code_objects

LINE = re.compile(r"^\s+(\S[^/]*?)\s*// ([0-9A-F]+):[^<]*(?:<[^+>]+(?:\+0x([0-9a-f]+))?>)?")
WRITES = ("ds_write", "ds_add", "ds_sub", "ds_min", "ds_max", "ds_and", "ds_or", "ds_xor", "ds_inc", "ds_dec", "ds_wrxchg", "ds_cmpst")
NONE = 1 << 30


def kernels_of(listing):
    """Name -> [(offset, instruction, offset of a branch's target or None)] of a disassembly."""
    out, base = {}, 0
    for line in listing.splitlines():
        head = re.match(r"^([0-9a-f]+) <(\S+)>:", line)
        if head:
            base, code = int(head.group(1), 16), []
            out[head.group(2)] = code
            continue
        m = LINE.match(line)
        if m:
            target = int(m.group(3) or "0", 16) if m.group(1).startswith(("s_cbranch", "s_branch")) else None
            code.append((int(m.group(2), 16) - base, m.group(1), target))
    return out


def unwaited(code):
    """Offsets of the barriers that some way through the code reaches with an LDS write that no wait has covered. LDS
    instructions end in order, so the state is how many followed the last write that may be under way."""
    at = {off: i for i, (off, _, _) in enumerate(code)}
    state, work, bad = {0: NONE}, [0], set()
    while work:
        i = work.pop()
        after = state[i]
        off, text, target = code[i]
        op = text.split()[0]
        assert not op.startswith(("s_setpc", "s_swappc", "s_call", "s_cbranch_g")), text
        if op.startswith("ds_"):
            after = 0 if op.startswith(WRITES) else (after + 1 if after < NONE else NONE)
        elif op == "s_waitcnt":
            m = re.search(r"lgkmcnt\((\d+)\)", text)
            if m and int(m.group(1)) <= after:
                after = NONE
        elif op == "s_barrier" and after < NONE:
            bad.add(off)
        follow = [] if op in ("s_endpgm", "s_branch") else [i + 1]
        if target is not None:
            follow.append(at[target])
        for n in follow:
            if n < len(code) and after < state.get(n, NONE + 1):
                state[n] = after
                work.append(n)
    return sorted(bad)


def test_walk():
    """A write before the barrier; one waited for; one that only a loop brings back to its head; a wait for all but the newest."""
    def code(*lines):
        return [(4 * i, *(x if isinstance(x, tuple) else (x, None))) for i, x in enumerate(lines)]

    assert unwaited(code("ds_write_b32 v0, v1", "s_barrier", "s_endpgm")) == [4]
    assert unwaited(code("ds_write_b32 v0, v1", "s_waitcnt lgkmcnt(0)", "s_barrier", "s_endpgm")) == []
    loop = ["s_nop 0", "s_waitcnt vmcnt(0)", "s_barrier", "ds_write_b32 v0, v1", ("s_cbranch_scc1 65532", 4), "s_endpgm"]
    assert unwaited(code(*loop)) == [8]
    loop[1] = "s_waitcnt vmcnt(0) lgkmcnt(0)"
    assert unwaited(code(*loop)) == []
    assert unwaited(code("ds_write_b32 v0, v1", "ds_read_b32 v2, v3", "s_waitcnt lgkmcnt(1)", "s_barrier", "s_endpgm")) == []
    assert unwaited(code("ds_read_b32 v2, v3", "ds_write_b32 v0, v1", "s_waitcnt lgkmcnt(1)", "s_barrier", "s_endpgm")) == [12]
    assert unwaited(code(("s_cbranch_scc1 1", 8), "ds_write_b32 v0, v1", "s_barrier", "s_endpgm")) == [8]


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    tool = os.path.join(os.path.dirname(os.path.realpath(B.HIPCC)), "..", "llvm", "bin", "llvm-objdump")
    tool = tool if os.path.exists(tool) else shutil.which("llvm-objdump")
    if not tool:
        pytest.skip("no llvm-objdump beside hipcc")
    with open(sv.LIB_PATH, "rb") as f:
        data = f.read()
    found = {}
    for i, elf in enumerate(code_objects(data)):
        path = tmp_path_factory.mktemp("code") / f"{i}.elf"
        path.write_bytes(elf)
        found.update(kernels_of(subprocess.run([tool, "-d", str(path)], capture_output=True, text=True, check=True).stdout))
    return found


def test_every_kernel(built):
    assert len(built) > 100
    assert sum(text.startswith("s_barrier") for code in built.values() for _, text, _ in code) > 1000
    bad = {name: unwaited(code) for name, code in built.items()}
    assert {name: offs for name, offs in bad.items() if offs} == {}
