"""The built kernels' instructions, on the CPU: wait states that the compiler counts only
for instructions that it knows, not for those inside assembly in the source.

A vector instruction's scalar result may be read by a memory instruction five wait states
later at the earliest, and the sums of a 32 x 32 matrix instruction by one that is none after
its passes (four cycles each: 8 for 16 products of 16 bits, 16 for 2 of float32) and four, or
two, more.  A wait state is an instruction, or n + 1 of them with
``s_nop n``; every way to an instruction is followed back, over branches too.
"""
import collections
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(HERE), "paper_2607_19456_amd", "libdecode_attn.so")
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"

pytestmark = [
    pytest.mark.skipif(not os.path.exists(LIB), reason="HIP library not built"),
    pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs llvm-objdump")]

REGISTER = re.compile(r"\b([sva])(\d+)\b|\b([sva])\[(\d+):(\d+)\]|\b(vcc)\b")
MEMORY = ("buffer_", "global_", "flat_", "scratch_")

# address, name, operands (texts), address of a branch's target or None
Instruction = collections.namedtuple("Instruction", "at name operands target")


def registers(text, kinds):
    """The registers of these kinds that an operand names."""
    out = set()
    for m in REGISTER.finditer(text):
        if m[6]:
            if "s" in kinds:
                out.add("vcc")
        elif (m[1] or m[3]) in kinds:
            out |= {m[1] + m[2]} if m[1] else {m[3] + str(i) for i in range(int(m[4]), int(m[5]) + 1)}
    return out


def parse(text):
    """{kernel's name: its instructions} of a disassembly."""
    out, now = {}, None
    for line in text.splitlines():
        label = re.match(r"(?:[0-9a-f]+ )?<(.+)>:$", line)
        if label:
            now = out.setdefault(label[1], [])
            continue
        code, _, note = line.partition("//")
        word = code.split(None, 1)
        if now is None or not line.startswith("\t") or not word or ":" not in note:
            continue
        target = re.search(r"<.*\+0x([0-9a-f]+)>", note)
        now.append(Instruction(int(note.split(":")[0], 16), word[0],
                               [x.strip() for x in word[1].split(",")] if len(word) > 1 else [],
                               int(target[1], 16) if target else None))
    return {name: x for name, x in out.items() if x}


def before(code):
    """For each instruction, the indexes of those that may come right before it."""
    index = {x.at: i for i, x in enumerate(code)}
    out = [[] for _ in code]
    for i, x in enumerate(code):
        if x.name.startswith(("s_branch", "s_cbranch")) and x.target is not None:
            to = index.get(code[0].at + x.target)
            if to is not None:
                out[to].append(i)
        if i + 1 < len(code) and x.name not in ("s_branch", "s_endpgm", "s_setpc_b64"):
            out[i + 1].append(i)
    return out


def search(code, ways, i, most, found):
    """(wait states between, instruction) of those that found() holds for on the ways back
    from i, less than `most` states far; a way ends there."""
    out, seen, open_ = [], {}, [(j, 0) for j in ways[i]]
    while open_:
        j, w = open_.pop()
        if w >= most or seen.get(j, most) <= w:
            continue
        seen[j] = w
        x = code[j]
        if found(x):
            out.append((w, x))
            continue
        w += int(x.operands[0], 0) + 1 if x.name == "s_nop" else 1
        open_ += [(y, w) for y in ways[j]]
    return out


def scalar_results(x):
    """Scalar registers that a vector instruction writes."""
    if not x.name.startswith("v_"):
        return set()
    n = 2 if "_co_" in x.name or "div_scale" in x.name else 1
    return set().union(*(registers(y, "s") for y in x.operands[:n])) if x.operands else set()


def scalars_too_early(code):
    """Memory instructions that read a vector instruction's scalar result too early."""
    ways, out = before(code), []
    for i, x in enumerate(code):
        if not x.name.startswith(MEMORY):
            continue
        reads = set().union(*(registers(y, "s") for y in x.operands)) if x.operands else set()
        if reads:
            out += [(x, w, y) for w, y in
                    search(code, ways, i, 5, lambda y: scalar_results(y) & reads)]
    return out


SUMS = {"v_mfma_f32_32x32x16_bf16": 12, "v_mfma_f32_32x32x16_f16": 12, "v_mfma_f32_32x32x2_f32": 18}


def sums_too_early(code):
    """Instructions other than products that read, or write over, a product's sums too early."""
    ways, out = before(code), []
    for i, x in enumerate(code):
        if x.name.startswith("v_mfma") or not x.name.startswith(("v_", "ds_") + MEMORY):
            continue
        uses = set().union(*(registers(y, "va") for y in x.operands)) if x.operands else set()
        out += [(x, w, y) for w, y in
                search(code, ways, i, max(SUMS.values()),
                       lambda y: y.name in SUMS and registers(y.operands[0], "va") & uses)
                if w < SUMS[y.name]]
    return out


def said(bad):
    return "\n".join(f"{name}: {x.name} {x.operands} at {x.at:#x}, {w} wait states after {y.name} "
                     f"{y.operands}" for name, b in bad.items() for x, w, y in b[:5])


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """All kernels of the library."""
    where = tmp_path_factory.mktemp("code")
    copy = str(where / "lib.so")
    shutil.copy(LIB, copy)
    subprocess.run([OBJDUMP, "--offloading", copy], cwd=where, check=True, capture_output=True)
    out = {}
    for name in sorted(os.listdir(where)):
        if "gfx950" in name:
            dis = subprocess.run([OBJDUMP, "-d", "--no-leading-addr", name], cwd=where, check=True,
                                 capture_output=True, text=True)
            out.update(parse(dis.stdout))
    assert sum("prompt_" in x for x in out) > 50 and len(out) > 200
    return out


def test_scalar_registers_are_written_in_time(kernels):
    bad = {name: scalars_too_early(code) for name, code in kernels.items()}
    bad = {name: x for name, x in bad.items() if x}
    assert not bad, said(bad)


def test_sums_are_there_when_they_are_read(kernels):
    """Of the kernels whose products are in assembly."""
    bad = {name: sums_too_early(code) for name, code in kernels.items() if "prompt_" in name}
    bad = {name: x for name, x in bad.items() if x}
    assert not bad, said(bad)


EARLY = """
0000000000001000 <kernel>:
\tv_readlane_b32 s16, v252, 16                               // 000000001000: D2890010 000121FC
\ts_mov_b32 m0, s69                                          // 000000001008: BEFC0045
\ts_nop {nop}                                                    // 00000000100C: BF800000
\tbuffer_load_dwordx4 v188, s[8:11], s16 offen lds           // 000000001010: E05D1000 100200BC
\ts_cbranch_scc0 65532                                       // 000000001018: BF84FFFC <kernel+{to}>
\ts_endpgm                                                   // 00000000101C: BF810000
"""


def test_what_the_search_finds():
    """Two states are too few, five enough; and over a branch back to the load."""
    (code,) = parse(EARLY.format(nop=0, to="0x0")).values()
    ((x, w, y),) = scalars_too_early(code)
    assert (x.at, w, y.name) == (0x1010, 2, "v_readlane_b32")
    (code,) = parse(EARLY.format(nop=3, to="0x0")).values()
    assert not scalars_too_early(code)
    code = code[1:] + [code[0]._replace(at=0x1020)]
    code = [x._replace(target=0x8) if x.target is not None else x for x in code]
    code[-2:] = [code[-1]._replace(at=0x101c), Instruction(0x1020, "s_branch", [], 0x8)]
    ((x, w, y),) = scalars_too_early(code)          # the branch alone lies between
    assert (x.at, w) == (0x1010, 1)
    sums = """
0000000000001000 <kernel>:
\tv_mfma_f32_32x32x2_f32 a[0:15], v5, v2, a[0:15]            // 000000001000: D3C48000 04020505
\ts_nop {nop}                                                   // 000000001008: BF80000F
\tv_accvgpr_read_b32 v22, a15                                // 00000000100C: D3D84016 1800010F
\ts_endpgm                                                   // 000000001014: BF810000
"""
    (code,) = parse(sums.format(nop=16)).values()
    assert [(x.at, w) for x, w, _ in sums_too_early(code)] == [(0x100c, 17)]
    (code,) = parse(sums.format(nop=17)).values()
    assert not sums_too_early(code)
