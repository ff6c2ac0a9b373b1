"""Loads into LDS in inline assembly take their windows from scalar registers and their place from m0.  A scalar register that a vector instruction has written is
read by such a load five states later at the earliest, m0 that a scalar one has written one state later; the compiler sees to that in its own code only.  These
tests compile the kernels for gfx950 and follow the registers through the assembly."""
import concurrent.futures
import os
import re
import subprocess

import pytest

from paper_2311_01282_amd import build
from tests.test_prefill_code_host import Code

pytestmark = pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")
SOURCES = ["fd_kv_prefill_kernels", "fd_latent_kernels", "fd_latent_prefill_kernels", "fd_nibble_kernels", "fd_prefill_kernels"]
LOAD = re.compile(r"(buffer_load|global_load_lds)")
STATES = 5


def registers(text):
    out = set()
    for first, last in re.findall(r"\bs\[(\d+):(\d+)\]", text):
        out.update(range(int(first), int(last) + 1))
    out.update(int(n) for n in re.findall(r"\bs(\d+)\b", text))
    if re.search(r"\bm0\b", text):
        out.add("m0")
    return out


def too_early(code):
    """Loads in inline assembly that read a scalar register too soon after it was written, over all paths; and how many such loads there are."""
    entry = [None] * len(code.blocks)            # register -> states that are still to pass
    entry[0] = {}
    found, loads, todo = set(), set(), [0]
    while todo:
        i = todo.pop()
        left = dict(entry[i])
        for at, (ins, inline) in enumerate(code.blocks[i]):
            op, _, args = ins.partition(" ")
            written, _, read = args.partition(",")
            if inline and LOAD.match(op):
                loads.add((i, at))
                if (registers(args) | {"m0"}) & set(left):
                    found.add((i, at))
            passed = int(args, 0) + 1 if op == "s_nop" else 1
            left = {r: n - passed for r, n in left.items() if n > passed}
            if op.startswith(("v_readfirstlane", "v_readlane", "v_cmp")):
                left.update((r, STATES) for r in registers(written))
            elif op.startswith("s_") and written.strip() == "m0" and read:
                left["m0"] = max(left.get("m0", 0), 1)
        for j in code.next[i]:
            merged = dict(entry[j] or {})
            for r, n in left.items():
                merged[r] = max(merged.get(r, 0), n)
            if entry[j] is None or merged != entry[j]:
                entry[j] = merged
                todo.append(j)
    return found, len(loads)


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    to = tmp_path_factory.mktemp("assembly")

    def one(name):
        path = str(to / (name + ".s"))
        subprocess.check_call([build.hipcc()] + build.FLAGS + ["-w", "--cuda-device-only", "-S", os.path.join(build.CSRC, name + ".hip"), "-o", path],
                              stderr=subprocess.DEVNULL)
        return open(path).read()
    with concurrent.futures.ThreadPoolExecutor(max_workers=4) as pool:
        return dict(zip(SOURCES, pool.map(one, SOURCES)))


@pytest.mark.parametrize("source", SOURCES)
def test_registers_have_settled(assembly, source):
    text, loads = assembly[source], 0
    names = re.findall(r"^\s*\.amdhsa_kernel (\S+)", text, re.M)
    assert names
    for name in names:
        found, n = too_early(Code(text, re.escape(name)))
        assert not found, (name, sorted(found)[:4])
        loads += n
    assert loads > 0


def test_what_it_finds():
    def code(*lines):
        return Code("kernel:\n" + "\n".join(lines) + "\n.Lfunc_end0:\n", "kernel")
    load = ["\t;#ASMSTART", "\ts_nop 0", "\tbuffer_load_dwordx4 v1, s[4:7], 0 offen lds", "\t;#ASMEND"]
    write = "\tv_readfirstlane_b32 s5, v0"
    assert len(too_early(code(write, *load))[0]) == 1
    assert len(too_early(code(write, "\ts_nop 2", *load))[0]) == 1
    assert not too_early(code(write, "\ts_nop 3", *load))[0]
    assert not too_early(code("\tv_readfirstlane_b32 s8, v0", *load))[0]
    assert len(too_early(code(write, "\ts_cbranch_scc0 .LBB0_1", "\ts_nop 4", ".LBB0_1:", *load))[0]) == 1
    assert not too_early(code("\ts_mov_b32 m0, s1", *load))[0]
    assert len(too_early(code("\ts_mov_b32 m0, s1", load[0], *load[2:]))[0]) == 1
