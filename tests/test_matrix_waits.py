"""What the compiler cannot know of the matrix instructions that vocab_kernels.h writes out: the waits around them.  The built library's own
code is listed and every way that leads to such an instruction is looked at: no vector instruction may write one of its operands in the two
wait states before it, and none may touch its sums before they have arrived."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2104_11125_amd import build

BEFORE = 2                      # wait states from a vector instruction's result to a matrix instruction that reads it
BEHIND = 18                     # and from a matrix instruction of at most 16 passes to another that reads or writes its sums
LINE = re.compile(r"^\s+(\S+)\s*(.*?)\s*// ([0-9A-F]+):((?: [0-9A-F]{8})+)(?: <.*>)?$")


def _registers(text):
    """The vector and accumulation registers that an operand names."""
    found = set()
    for kind, one, first, last in re.findall(r"\b([va])(?:(\d+)\b|\[(\d+):(\d+)\])", text):
        for i in range(int(one or first), int(one or last) + 1):
            found.add((kind, i))
    return found


def _instructions(listing):
    """(address, name, operands, targets): every instruction of a function and where it may go on."""
    code = []
    for line in listing:
        m = LINE.match(line)
        if not m:
            continue
        name, operands, at, words = m.group(1), m.group(2).split(", "), int(m.group(3), 16), m.group(4).split()
        ahead = at + 4 * len(words)
        if name == "s_endpgm":
            targets = []
        elif name.startswith(("s_branch", "s_cbranch")):
            jump = int(words[0], 16) & 0xffff
            to = ahead + 4 * (jump - 0x10000 if jump >= 0x8000 else jump)
            targets = [to] if name == "s_branch" else [ahead, to]
        else:
            assert not name.startswith(("s_setpc", "s_swappc", "s_call", "s_cbranch_i")), name
            targets = [ahead]
        code.append((at, name, operands, targets))
    return code


def _states(name, operands):
    return int(operands[0]) + 1 if name == "s_nop" else 1


def _behind(code, before, index, states):
    """Every instruction that may be executed fewer than `states` wait states before instruction `index`."""
    seen, todo, found = {}, [(i, 0) for i in before[index]], set()
    while todo:
        i, passed = todo.pop()
        if passed >= states or seen.get(i, states) <= passed:
            continue
        seen[i] = passed
        found.add(i)
        todo += [(j, passed + _states(*code[i][1:3])) for j in before[i]]
    return found


def missing_waits(listing):
    code = _instructions(listing)
    index = {at: i for i, (at, *_) in enumerate(code)}
    before, todo, seen = [[] for _ in code], [0], {0}
    while todo:                                             # what can be reached
        i = todo.pop()
        for to in (index[t] for t in code[i][3]):
            before[to].append(i)
            if to not in seen:
                seen.add(to)
                todo.append(to)
    faults = []
    for i, (at, name, operands, _) in enumerate(code):
        if name.startswith("v_mfma"):
            reads = set().union(*map(_registers, operands[1:4]))
            for j in _behind(code, before, i, BEFORE):
                _, other, to, _ = code[j]
                if other.startswith("v_") and not other.startswith("v_mfma") and _registers(to[0]) & reads:
                    faults.append((hex(at), other, to))
        elif name.startswith(("v_", "ds_", "global_", "flat_", "scratch_", "buffer_")):
            touched = {r for r in set().union(*map(_registers, operands)) if r[0] == "a"}
            if touched:
                faults += [(hex(at), name, operands) for j in _behind(code, before, i, BEHIND)
                           if code[j][1].startswith("v_mfma") and _registers(code[j][2][0]) & touched]
    return faults, sum(name.startswith("v_mfma") for _, name, _, _ in code)


def _listing(*lines):
    """Instructions of one word each, as the tool prints them; a number behind a branch is where it goes, in instructions from it."""
    return [f"\t{text.split('@')[0]} // {4 * i:012X}: BF82{int(text.split('@')[1]) & 0xffff if '@' in text else 0:04X}" for i, text in enumerate(lines)]


PRODUCT = "v_mfma_f32_16x16x32_bf16 a[4:7], v[8:11], v[0:3], a[4:7]"


@pytest.mark.parametrize("lines,faults", [
    (["v_mov_b32_e32 v9, v20", PRODUCT, "s_endpgm"], 1),
    (["v_mov_b32_e32 v9, v20", "s_mov_b32 s0, 0", PRODUCT, "s_endpgm"], 1),
    (["v_mov_b32_e32 v9, v20", "s_nop 1", PRODUCT, "s_endpgm"], 0),
    (["v_mov_b32_e32 v12, v20", PRODUCT, "s_endpgm"], 0),
    (["ds_read_b128 v[8:11], v20", "s_waitcnt lgkmcnt(0)", PRODUCT, "s_endpgm"], 0),
    (["v_accvgpr_write_b32 a5, 0", PRODUCT, "s_endpgm"], 1),
    ([PRODUCT, "v_accvgpr_read_b32 v1, a6", "s_endpgm"], 1),
    ([PRODUCT, "s_nop 15", "v_accvgpr_read_b32 v1, a6", "s_endpgm"], 1),
    ([PRODUCT, "s_nop 15", "s_nop 15", "v_accvgpr_read_b32 v1, a6", "s_endpgm"], 0),
    # behind the end of a loop, at its beginning; the way past the loop is far enough
    ([PRODUCT, "s_nop 0", "v_mov_b32_e32 v2, v20", "s_cbranch_scc1 L@-4", "s_endpgm"], 1),
    (["s_branch L@1", "v_mov_b32_e32 v2, v20", PRODUCT, "s_endpgm"], 0)])
def test_the_check_itself(lines, faults):
    found, products = missing_waits(_listing(*lines))
    assert len(found) == faults and products == 1, found


def test_products_of_large_tiles(tmp_path):
    if not os.path.exists(build.LIB):
        build.build_library()
    tool = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"
    library = shutil.copy(build.LIB, tmp_path)
    subprocess.run([tool, "--offloading", library], cwd=tmp_path, check=True, capture_output=True)
    image, = [f for f in os.listdir(tmp_path) if f.endswith("gfx950")]
    text = subprocess.run([tool, "-d", image], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
    functions = re.split(r"^[0-9a-f]+ <(\S+)>:\n", text, flags=re.M)
    large = {name: body for name, body in zip(functions[1::2], functions[2::2]) if re.search(r"k_vocab_.*VocabConfigILi2ELi2ELi8ELi8E", name)}
    assert len(large) == 6                                  # sums, dz in one plane and in three, dx, dw in either type
    for name, body in large.items():
        faults, products = missing_waits(body.splitlines())
        assert products == 256 and "v_mfma_f32_16x16x32_bf16 a[" in body, name
        assert not faults, (name, faults[:5])
