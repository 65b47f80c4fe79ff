"""The vocabulary loss's large tile issues its matrix instructions from inline assembly, so that its 256 accumulators stay where they are; the compiler keeps no
distances for those.  A register that a vector instruction writes may be read by a matrix instruction two wait states later, and the result of a
16 x 16 x 32 product by anything but the next product into it 18 later.  Both are looked up in the built library, over loops' back edges too, and that nothing
moves an accumulator inside the stage loop."""
import os
import re
import subprocess

import pytest

from paper_2602_01410_amd import snip
from test_wait_states import OBJDUMP, code_objects

BEFORE, BEHIND = 2, 18


def registers(tok):
    m = re.fullmatch(r"([av])\[(\d+):(\d+)\]", tok)
    if m:
        return {(m[1], i) for i in range(int(m[2]), int(m[3]) + 1)}
    m = re.fullmatch(r"([av])(\d+)", tok)
    return {(m[1], int(m[2]))} if m else set()


def states(ins):
    return 1 + int(ins[1], 0) if ins[0] == "s_nop" else 1


def writes(ins):
    """Vector registers that an instruction of the vector unit (no memory) writes."""
    return registers(ins[1]) if ins[0].startswith("v_") and not ins[0].startswith("v_cmp") and len(ins) > 1 else set()


def pairs(seq):
    """(wait states between, earlier, later) of matrix instructions that come too soon, or whose results are taken too soon, in a run of instructions."""
    found = []
    for i, ins in enumerate(seq):
        product = ins[0].startswith("v_mfma")
        reads = set().union(*(registers(t) for t in (ins[2:] if ins[0].startswith("v_") else ins[1:])))
        need, waited = (BEFORE if product else BEHIND), 0
        for j in range(i - 1, -1, -1):
            old = seq[j]
            if waited >= need or old[0] in ("s_branch", "s_endpgm", "s_setpc_b64"):
                break
            if old[0].startswith("v_mfma") != product and writes(old) & (reads | writes(ins)):
                found.append((waited, " ".join(old), " ".join(ins)))
                break
            waited += states(old)
    return found


def kernels(lines):
    """Kernel of the large tile -> [(address, instruction)]."""
    found, body = {}, None
    for line in lines:
        m = re.match(r"([0-9a-f]+) <(\S+)>:", line)
        if m:
            body = found.setdefault(m[2], []) if "product_kernel" in m[2] and "TileILi256E" in m[2] else None
            continue
        if body is None or "//" not in line:
            continue
        text, note = line.split("//", 1)
        at = re.match(r"\s*([0-9A-Fa-f]+):", note)
        ins = [t.rstrip(",") for t in text.split()]
        if at and ins:
            body.append((int(at[1], 16), ins, note))
    return found


def back_edges(body):
    """(place of a branch backwards, place that it goes to)."""
    place, edges = {at: i for i, (at, _, _) in enumerate(body)}, []
    for i, (at, ins, _) in enumerate(body):
        if ins[0].startswith(("s_cbranch", "s_branch")):
            off = int(ins[1])
            to = at + 4 + 4 * (off - 65536 if off >= 32768 else off)
            if to <= at:
                edges.append((i, place[to]))
    return edges


def test_scan_finds_what_is_too_close():
    mfma = "v_mfma_f32_16x16x32_bf16 a[0:3] v[0:3] v[4:7] a[0:3]".split()
    assert [w for w, *_ in pairs(["v_add_u32 v4 v9 v9".split(), "s_nop 0".split(), mfma])] == [1]
    assert pairs(["v_add_u32 v4 v9 v9".split(), "s_nop 1".split(), mfma]) == []
    assert [w for w, *_ in pairs([mfma, "s_nop 15".split(), "v_accvgpr_read_b32 v9 a3".split()])] == [16]
    assert pairs([mfma, "s_nop 15".split(), "s_nop 1".split(), "v_accvgpr_read_b32 v9 a3".split()]) == []
    assert [w for w, *_ in pairs([mfma, "global_store_dword v8 a2 s[0:1]".split()])] == [0]


def test_library(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    seen, loops, found, moved = 0, 0, [], []
    for i, obj in enumerate(code_objects(snip.LIB_PATH)):
        if b"product_kernel" not in obj:
            continue
        path = tmp_path / f"{i}.co"
        path.write_bytes(obj)
        out = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True, timeout=300).stdout
        for name, body in kernels(out.splitlines()).items():
            seen += 1
            seq = [ins for _, ins, _ in body]
            found += [(name, *p) for p in pairs(seq)]
            for end, start in back_edges(body):
                found += [(name, *p) for p in pairs(seq[max(0, end - 40):end] + seq[start:start + 40])]
                loop = seq[start:end]
                products = [k for k, ins in enumerate(loop) if ins[0].startswith("v_mfma")]
                if products:
                    loops += 1
                    moved += [(name, " ".join(ins)) for ins in loop[products[0]:products[-1]] if "accvgpr" in ins[0]]
    assert seen == 4 and loops >= 4
    assert not found, (len(found), found[:5])
    assert not moved, (len(moved), moved[:5])
