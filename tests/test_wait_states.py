"""The built library's matrix instructions and what reads their results (no GPU).

The hardware does not hold back a reader of a matrix instruction's result: a
number of wait states have to pass (an instruction is one, s_nop n is n + 1), on
every path from the one to the other.  The compiler puts them in, but where paths
join behind a short branch it counts along one of them and may leave too few:
scores of fp32 attention rows past 128 entries lost their last product so.  This
follows every path through the disassembly of the library built here."""
import itertools
import os
import re
import shutil
import subprocess

import pytest

from paper_2605_19150_amd import pdssm

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
# wait states before a vector instruction or a store reads the result: passes + 2 for the fp32 instructions, passes + 4 for those of 16 bits
NEED = {"f32_16x16x4_f32": 10, "f32_32x32x2_f32": 18, "f32_32x32x1_2b_f32": 18, "f32_16x16x32_bf16": 8, "f32_32x32x16_bf16": 12}
STORES = ("ds_write", "ds_add", "ds_max", "buffer_store", "global_store", "flat_store", "scratch_store", "global_atomic")


def _regs(text):
    out = set()
    for kind, lo, hi in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        out |= {kind + str(k) for k in range(int(lo), int(hi) + 1)}
    return out | {kind + n for kind, n in re.findall(r"\b([va])(\d+)\b", text)}


def _operands(text):
    return re.split(r",\s*(?![^\[]*\])", text)


def _accesses(op, text):
    """(registers written, registers read) of an instruction of a lane."""
    if op.startswith(STORES):
        return set(), _regs(text)
    if not op.startswith(("v_", "ds_", "buffer_", "global_", "flat_", "scratch_")):
        return set(), set()
    first, rest = _regs(_operands(text)[0]), _regs(",".join(_operands(text)[1:]))
    if op.startswith("v_cmpx") or op.startswith("v_swap"):
        return first, first | rest
    if op.startswith(("v_fmac", "v_mac", "v_dot")):
        return first, first | rest
    return first, rest


def functions(lines):
    """Of each kernel with matrix instructions in the lines of a disassembly: (name, [(op, operands, index of the target or
    None)])."""
    name, body = None, []
    for line in itertools.chain(lines, ["<>:"]):
        if line.startswith("\t") and "//" in line:
            body.append(line)
        elif line.startswith("<"):
            if any("v_mfma" in x for x in body):
                yield name, _parse(body)
            name, body = line.rstrip()[1:-2], []


def _parse(body):
    code, at = [], {}
    for line in body:
        what, _, where = line.partition("//")
        op, _, text = what.strip().partition(" ")
        to = re.search(r"<\S+?(?:\+0x([0-9a-f]+))?>\s*$", where) if op.startswith(("s_branch", "s_cbranch")) else None
        at[int(where.partition(":")[0], 16)] = len(code)
        code.append((op, text, to and int(to[1] or "0", 16)))
    base = min(at)
    return [(op, text, None if to is None else at[base + to]) for op, text, to in code]


def too_early(code):
    """[(index of a matrix instruction, index of the reader, wait states between them)]"""
    touch = {}  # of the instructions that are reached
    found = []
    for k, (op, text, _) in enumerate(code):
        if not op.startswith("v_mfma"):
            continue
        need, todo, best = NEED[op[len("v_mfma_"):]], [(k + 1, 0, frozenset(_regs(_operands(text)[0])))], {}
        while todo:
            p, n, live = todo.pop()
            if p >= len(code) or n >= need or not live or best.get((p, live), need) <= n:
                continue
            best[p, live] = n
            op2, text2, to = code[p]
            if op2 == "s_endpgm":
                continue
            if op2 == "s_nop":
                n += int(text2, 0)
            elif op2.startswith("v_mfma"):  # the sum goes on in it, or it reads the result as a factor
                parts = _operands(text2)
                if _regs(",".join(parts[1:3])) & live:
                    found.append((k, p, n))
                live -= _regs(parts[0])
            else:
                if p not in touch:
                    touch[p] = set.union(*_accesses(op2, text2))
                if touch[p] & live:
                    found.append((k, p, n))
                    continue
            if to is not None:
                todo.append((to, n + 1, live))
            if op2 != "s_branch":
                todo.append((p + 1, n + 1, live))
    return found


def _listing(lines):
    text, at = ["<kernel>:"], 0
    places, out = {}, []
    for line in lines:
        if line.endswith(":"):
            places[line[:-1]] = at
        else:
            out.append((line, at))
            at += 4
    for line, pos in out:
        op, _, rest = line.partition(" ")
        to = " <kernel+0x%x>" % places[rest] if rest in places else ""
        text.append("\t%s %s // %012X: 00000000%s" % (op, "1" if to else rest, pos, to))
    return text


MFMA = "v_mfma_f32_16x16x4_f32 a[0:3], v1, v2, a[0:3]"


@pytest.mark.parametrize("lines,states", [
    ([MFMA, "s_nop 9", "v_accvgpr_read_b32 v5, a3"], None),
    ([MFMA, "s_nop 8", "v_accvgpr_read_b32 v5, a3"], 9),
    # a loop that is long enough, and the branch past it that is not
    ([MFMA, "s_cbranch_execz out", "loop:", *["v_mul_f32_e32 v7, v7, v8"] * 12, "s_cbranch_execnz loop", "out:", "s_or_b64 exec, exec, s[2:3]",
      "v_accvgpr_read_b32 v5, a3"], 2),
    ([MFMA, "s_cbranch_execz out", *["v_mul_f32_e32 v7, v7, v8"] * 12, "out:", "s_nop 7", "s_nop 0", "v_accvgpr_read_b32 v5, a3"], None),
    ([MFMA, MFMA, "s_nop 9", "global_store_dwordx4 v[8:9], a[0:3], off"], None),
    ([MFMA, "v_mov_b32_e32 v1, 0", "v_accvgpr_write_b32 a2, v1"], 1),
    ([MFMA, "v_mfma_f32_16x16x4_f32 a[4:7], v1, a2, a[4:7]", "s_endpgm "], 0)], ids=range(7))
def test_paths_are_followed(lines, states):
    (_, code), = functions(_listing(lines + ["s_endpgm "]))
    got = too_early(code)
    assert [n for _, _, n in got] == ([] if states is None else [states])


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_the_built_library(tmp_path):
    if not os.path.exists(pdssm.lib_path()):
        from paper_2605_19150_amd.build import build_library
        build_library()
    shutil.copy(pdssm.lib_path(), tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    kernels, bad = 0, []
    for f in sorted(tmp_path.glob("*gfx950*")):
        with subprocess.Popen([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", f.name], cwd=tmp_path, text=True,
                              stdout=subprocess.PIPE) as listing:
            for name, code in functions(listing.stdout):
                kernels += 1
                bad += ["%s: %s %s, %d states, %s %s" % (name, *code[k][:2], n, *code[p][:2]) for k, p, n in too_early(code)]
        assert listing.returncode == 0
    assert kernels > 60  # the scans alone
    assert not bad, "\n".join(bad)
