"""What the compiled kernels have to keep of their source (CPU only: the library's gfx950 code, disassembled).

Loads that go straight into LDS are counted by the wave that issued them alone.  A tile that all waves share can be
read after a barrier only if every wave has waited for its own loads (vmcnt(0)) before it.
"""
import os
import re
import shutil
import struct
import subprocess

import pytest

from paper_2609_39819_amd import kvt

OBJDUMP = next((p for p in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump")) if p and os.path.exists(p)),
               None)
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(library):
    """The gfx950 code objects in a library's bundles."""
    at = library.find(MAGIC)
    while at >= 0:
        count = struct.unpack_from("<Q", library, at + len(MAGIC))[0]
        p = at + len(MAGIC) + 8
        for _ in range(count):
            offset, size, n = struct.unpack_from("<QQQ", library, p)
            triple = library[p + 24:p + 24 + n]
            p += 24 + n
            if b"gfx950" in triple and size:
                yield library[at + offset:at + offset + size]
        at = library.find(MAGIC, at + len(MAGIC))


def functions(tmp_path, wanted):
    """{name: [(address, instruction, branch target or None)]} of the kernels whose name holds `wanted`."""
    found = {}
    with open(kvt.LIB_PATH, "rb") as f:
        library = f.read()
    for i, obj in enumerate(code_objects(library)):
        if wanted.encode() not in obj:
            continue
        path = tmp_path / f"{i}.o"
        path.write_bytes(obj)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True,
                              check=True).stdout
        name, start = None, 0
        for line in text.splitlines():
            head = re.match(r"([0-9a-f]+) <(\S+)>:", line)
            if head:
                start, name = int(head.group(1), 16), head.group(2) if wanted in head.group(2) else None
                if name:
                    found[name] = []
                continue
            m = re.match(r"\s+(\S.*?)\s*//\s*([0-9A-Fa-f]+):(?:.*<\S+?\+0x([0-9a-f]+)>)?", line)
            if name and m:
                op = m.group(1)
                target = start + int(m.group(3), 16) if m.group(3) and op.startswith(("s_branch", "s_cbranch")) else None
                found[name].append((int(m.group(2), 16), op, target))
    return found


def unwaited(code):
    """Addresses of loads into LDS that some path reaches from earlier ones through a barrier without a wait before
    it: (loads in flight, barrier passed, waited for) along every path."""
    index = {a: i for i, (a, _, _) in enumerate(code)}
    seen, todo, bad = set(), [(0, "none", False)], set()
    while todo:
        at = todo.pop()
        if at in seen or at[0] >= len(code):
            continue
        seen.add(at)
        i, state, passed = at
        address, op, target = code[i]
        if "load_lds" in op:
            if state != "none" and passed:
                bad.add(address)
            state, passed = "flying", False
        elif op.startswith("s_waitcnt") and "vmcnt(0)" in op:
            state = "waited" if state == "flying" else state
        elif op.startswith("s_barrier"):
            state, passed = ("none", False) if state != "flying" else (state, True)
        if op.startswith("s_endpgm"):
            continue
        if target is not None:
            todo.append((index[target], state, passed))
        if not op.startswith("s_branch"):
            todo.append((i + 1, state, passed))
    return bad


@pytest.mark.skipif(OBJDUMP is None, reason="needs llvm-objdump")
@pytest.mark.parametrize("kernel", ["diff_extend_kernel", "extend_fwd_kernel"])
def test_loads_into_lds_are_waited_for_before_the_barrier(tmp_path, kernel):
    kernels = functions(tmp_path, kernel)
    kernels = {n: c for n, c in kernels.items() if any("load_lds" in op for _, op, _ in c)}
    assert kernels, f"no {kernel} with loads into LDS in {kvt.LIB_PATH}"
    for name, code in kernels.items():
        print(name, len(code), sum("load_lds" in op for _, op, _ in code), sum(op.startswith("s_barrier") for _, op, _ in code))
        assert all(t is not None for _, op, t in code if op.startswith(("s_branch", "s_cbranch")))
        assert not any(op.startswith(("s_setpc", "s_swappc")) for _, op, _ in code)
        assert not unwaited(code), name


def test_the_search_finds_a_missing_wait():
    load, wait, barrier, end = "global_load_lds_dwordx4 v1, s[0:1]", "s_waitcnt vmcnt(0)", "s_barrier", "s_endpgm"

    def code(*ops, back=None):
        rows = [(4 * i, op, None) for i, op in enumerate(ops)]
        if back is not None:
            rows[-2] = (rows[-2][0], "s_cbranch_scc1 -1", 4 * back)
        return rows
    good = code(load, wait, barrier, load, load, barrier, wait, barrier, "branch", end, back=3)
    assert not unwaited(good)
    assert unwaited(code(load, wait, barrier, load, barrier, "branch", end, back=3)) == {12}    # no wait
    assert unwaited(code(load, wait, barrier, load, barrier, wait, "branch", end, back=3)) == {12}   # too late
    skipped = code(load, wait, barrier, load, "s_cbranch_execz 1", wait, barrier, "branch", end, back=3)
    skipped[4] = (16, "s_cbranch_execz 1", 24)
    assert unwaited(skipped) == {12}                                                              # not on every path
