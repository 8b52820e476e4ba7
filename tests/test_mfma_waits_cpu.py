"""Matrix results are used only after the wait states they need, on every path through a kernel.

gfx950 does not hold an instruction back until a matrix product's result is there: the compiler has to
leave wait states between the product and the first instruction that reads or overwrites its result, 8 for
the 16x16x32 bf16 product and 10 for the 16x16x4 binary32 one.  The compiler of ROCm 7.2 leaves them out
where that first use stands behind a block that may be skipped.  So the sources have no condition between
a product and its use, and this test walks the assembly that they compile to.  No GPU is needed."""
import os
import re
import subprocess

import pytest

from paper_1906_07155_amd import build as B

NEEDS = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x4_f32": 10}
MOST = max(NEEDS.values())
ENDS = ("s_branch", "s_endpgm", "s_setpc", "s_swappc")
REGISTER = re.compile(r"\b([va])(?:(\d+)|\[(\d+):(\d+)\])")


def registers(text):
    out = set()
    for kind, one, low, high in REGISTER.findall(text):
        out.update((kind, i) for i in ([int(one)] if one else range(int(low), int(high) + 1)))
    return out


def functions(text):
    """{kernel: its labels (a string) and instructions (line, operation, operands)}"""
    out, name = {}, None
    for number, line in enumerate(text.splitlines(), 1):
        line = line.split(";")[0].rstrip()
        label = re.match(r"(\S+):\s*$", line)
        if label and label[1].startswith(".Lfunc_end"):
            name = None
        elif label and label[1].startswith(".LBB"):
            if name:
                out[name].append(label[1])
        elif label and not label[1].startswith("."):
            name = label[1]
            out[name] = []
        elif name and line.strip() and not line.strip().startswith("."):
            op, _, operands = line.strip().replace("\t", " ").partition(" ")
            out[name].append((number, op, operands.strip()))
    return out


def blocks_of(code):
    blocks = [(None, [])]
    for item in code:
        if isinstance(item, str):
            blocks.append((item, []))
        else:
            blocks[-1][1].append(item)
            if item[1].startswith("s_cbranch") or item[1].startswith(ENDS):
                blocks.append((None, []))
    index = {label: i for i, (label, _) in enumerate(blocks) if label}
    after = []
    for i, (_, items) in enumerate(blocks):
        end = items[-1] if items else (0, "", "")
        to = [index[end[2]]] if end[1].startswith(("s_cbranch", "s_branch")) else []
        if not end[1].startswith(ENDS) and i + 1 < len(blocks):
            to.append(i + 1)
        after.append(to)
    return blocks, after


def walk(items, state, found=None):
    """Through one block: ``state`` has, by register, (wait states since its product, line, operation)."""
    for line, op, operands in items:
        product = op.startswith("v_mfma")
        parts = [p.strip() for p in re.split(r",(?![^\[]*\])", operands)]
        if not op.startswith("s_"):
            # a product that goes on with a sum may read and write it at once
            used = registers(" ".join(parts[1:3])) if product else registers(operands)
            for r in used & state.keys():
                since, source, maker = state[r]
                if found is not None and since < NEEDS[maker]:
                    found.append(f"line {line}: {op} uses {r[0]}{r[1]} {since} wait states after {maker} of line {source}")
        states = int(operands, 0) + 1 if op == "s_nop" else 1
        for r, (since, *rest) in list(state.items()):
            if since + states >= MOST:
                del state[r]
            else:
                state[r] = (since + states, *rest)
        if product:
            assert op in NEEDS, f"line {line}: the wait states of {op} are not in the table"
            state.update(dict.fromkeys(registers(parts[0]), (0, line, op)))


def early_uses(text):
    found = []
    for name, code in functions(text).items():
        blocks, after = blocks_of(code)
        starts = [None] * len(blocks)
        starts[0], todo = {}, [0]
        while todo:                       # the least wait states on any path to a block
            i = todo.pop()
            state = dict(starts[i])
            walk(blocks[i][1], state)
            for to in after[i]:
                if starts[to] is None:
                    starts[to] = dict(state)
                    todo.append(to)
                    continue
                less = {r: v for r, v in state.items() if r not in starts[to] or v[0] < starts[to][r][0]}
                if less:
                    starts[to].update(less)
                    todo.append(to)
        for (_, items), state in zip(blocks, starts):
            if state is not None:
                here = []
                walk(items, dict(state), here)
                found += [f"{name}: {x}" for x in here]
    return found


@pytest.mark.parametrize("source", ["attn_bwd", "attn_dense", "attn_recall"])
def test_products_are_waited_for(source, tmp_path):
    path = os.path.join(os.path.dirname(B.__file__), "csrc", source + ".hip")
    out = tmp_path / (source + ".s")
    subprocess.check_call([B.HIPCC, *B.FLAGS, "--cuda-device-only", "-S", path, "-o", str(out)], stderr=subprocess.DEVNULL)
    text = out.read_text()
    assert any(op in text for op in NEEDS)
    assert early_uses(text) == []


PLANTED = """kernel:
\ts_cbranch_scc1 .LBB0_9
\tv_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], 0
\ts_cbranch_vccz .LBB0_2
; %bb.1:
\ts_nop 7
\tv_sub_f32_e32 v0, v0, v20
.LBB0_2:
{wait}\tv_mul_f32_e32 v1, v1, v2
.LBB0_9:
\ts_endpgm
.Lfunc_end0:
"""


@pytest.mark.parametrize("wait,early", [("", True), ("\ts_nop 5\n", True), ("\ts_nop 6\n", False)])
def test_the_walk_sees_what_a_skipped_block_hides(wait, early):
    assert bool(early_uses(PLANTED.format(wait=wait))) == early
