"""How long after a matrix instruction its result is read, in the kernels built here (CPU only).

The hardware does not hold an ordinary instruction back that reads a matrix instruction's result: as many wait states have to lie between the two, on
every way from one to the other, as the compiler keeps where there is one way only.  Where ways part and meet again behind a matrix instruction it follows
the first that it tries and may leave too few on a shorter one (experts_tile.h, sums_done), so the built code is looked at: every way from every
matrix instruction, through branches and round loops, to the first ordinary instruction that reads or writes what it wrote."""
import collections
import os
import re
import subprocess

import pytest

from paper_2305_08872_amd import build as hip_build
from test_kernel_resources import _tool

# What the compiler keeps between a matrix instruction and a reader of its result with nothing else between (results of 4 registers are there after
# 4 passes, those of 16 after 8, of fp32 operands after 16; a pass has four cycles, a wait state one issue).
STATES = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x32_f16": 8, "v_mfma_f32_32x32x16_bf16": 12, "v_mfma_i32_32x32x32_i8": 12,
          "v_mfma_scale_f32_16x16x128_f8f6f4": 12, "v_mfma_f32_32x32x2_f32": 18, "v_mfma_f64_16x16x4_f64": 19}
LINE = re.compile(r"^\s+(\S+)\s*(.*?)\s*// ([0-9A-F]+):(?:.*?<([^>]+)>)?")
REGISTER = re.compile(r"\b([av])(?:(\d+)|\[(\d+):(\d+)\])")


def _code(obj, tmp):
    bundle, code = os.path.join(tmp, "bundle"), os.path.join(tmp, "code")
    subprocess.check_call([_tool("llvm-objcopy"), "--dump-section", ".hip_fatbin=" + bundle, obj, os.devnull])
    subprocess.check_call([_tool("clang-offload-bundler"), "--type=o", "--unbundle", "--input=" + bundle, "--output=" + code,
                           "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"])
    return subprocess.check_output([_tool("llvm-objdump"), "-d", "--no-show-raw-insn", code], text=True)


def functions(listing):
    """(name, [(address, instruction, operands, branch target)])"""
    name, body = None, []
    for line in listing.splitlines():
        head = re.match(r"^[0-9a-f]+ <(.+)>:", line)
        if head:
            if name:
                yield name, body
            name, body = head.group(1), []
            continue
        m = LINE.match(line)
        if m and name:
            body.append((int(m.group(3), 16), m.group(1), m.group(2), m.group(4)))
    if name:
        yield name, body


def registers(text):
    out = set()
    for m in REGISTER.finditer(text):
        lo, hi = int(m.group(2) or m.group(3)), int(m.group(2) or m.group(4))
        out |= {(m.group(1), r) for r in range(lo, hi + 1)}
    return frozenset(out)


def operands(text):
    return [x.strip() for x in re.split(r",(?![^\[]*\])", text)] if text else []


def touched(op, text):
    """Registers that an ordinary vector or memory instruction reads or writes; of a matrix instruction those of its first two factors (its sums
    are the matrix cores' own to order)."""
    if op.startswith("v_mfma"):
        return registers(", ".join(operands(text)[1:3]))
    return registers(text) if op[0] in "vdgbf" else frozenset()


def distances(body):
    """{matrix instruction's name: (fewest wait states to an instruction that touches its result, that one's address)}"""
    at = {a: i for i, (a, *_rest) in enumerate(body)}
    start = body[0][0]
    after = []
    for i, (_a, op, _text, target) in enumerate(body):
        to = []
        if op.startswith(("s_cbranch", "s_branch")):
            to.append(at[start + (int(target.rsplit("+0x", 1)[1], 16) if "+0x" in target else 0)])
        if op not in ("s_branch", "s_endpgm", "s_setpc_b64") and i + 1 < len(body):
            to.append(i + 1)
        after.append(to)
    states = [int(text.split()[0], 0) + 1 if op == "s_nop" else 1 for _a, op, text, _t in body]
    uses = [touched(op, text) for _a, op, text, _t in body]
    least = {}
    for i, (_a, op, text, _t) in enumerate(body):
        if not op.startswith("v_mfma"):
            continue
        result, enough = registers(operands(text)[0]), STATES[op]
        seen, todo = {}, [(j, 0) for j in after[i]]
        while todo:
            j, n = todo.pop()
            if n >= enough or seen.get(j, enough) <= n:
                continue
            seen[j] = n
            if uses[j] & result:
                if n < least.get(op, (enough, 0))[0]:
                    least[op] = (n, body[j][0])
                continue
            if body[j][1].startswith("v_mfma") and registers(operands(body[j][2])[0]) >= result:
                continue   # (written anew: that one has a way of its own)
            todo += [(k, n + states[j]) for k in after[j]]
    return least


def test_a_short_way_round_a_branch_is_seen():
    """Two ways from a matrix instruction to a reader, one with enough wait states; and one round a loop."""
    def body(*lines):
        return [(4 * i, line.split()[0], line.partition(" ")[2], "f+0x%x" % (4 * to) if to is not None else None) for i, (line, to) in enumerate(lines)]
    forward = [("v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[8:11]", None), ("s_cbranch_scc1 1", 3), ("s_nop 7", None), ("v_accvgpr_read_b32 v9, a3", None), ("s_endpgm", None)]
    assert distances(body(*forward)) == {"v_mfma_f32_16x16x32_bf16": (1, 12)}
    forward[1] = ("s_nop 0", None)
    assert distances(body(*forward)) == {}
    loop = [("s_nop 0", None), ("v_mov_b32 v9, v3", None), ("v_mfma_f32_16x16x32_bf16 v[0:3], v[16:19], v[4:7], v[0:3]", None), ("s_nop 4", None), ("s_cbranch_scc1 1", 1), ("s_endpgm", None)]
    assert distances(body(*loop)) == {"v_mfma_f32_16x16x32_bf16": (6, 4)}
    loop[3] = ("s_nop 6", None)
    assert distances(body(*loop)) == {}
    # (the sums of a following matrix instruction are not an ordinary reader, its factors are)
    chain = [loop[2], ("v_mfma_f32_16x16x32_bf16 v[0:3], v[16:19], v[4:7], v[0:3]", None), ("s_endpgm", None)]
    assert distances(body(*chain)) == {}
    chain[1] = ("v_mfma_f32_16x16x32_bf16 v[20:23], v[0:3], v[4:7], v[20:23]", None)
    assert distances(body(*chain)) == {"v_mfma_f32_16x16x32_bf16": (0, 4)}


# (the others' kernels have no matrix instructions)
@pytest.mark.parametrize("source", [s for s in hip_build.SOURCES if re.match(r"identity_|count_i8|valu_probe|mmlike_boost|experts_(mm|sums)|adapters_(down|up|outer)", s)])
def test_results_are_there_when_they_are_read(source, tmp_path):
    obj = os.path.join(hip_build.OBJ_DIR, os.path.splitext(source)[0] + ".o")
    if not os.path.exists(obj):
        hip_build.build()
    short = collections.OrderedDict()
    for name, body in functions(_code(obj, str(tmp_path))):
        for op, (n, where) in distances(body).items():
            short["%s: %s" % (name, op)] = "%d of %d wait states before %x" % (n, STATES[op], where)
    assert not short
