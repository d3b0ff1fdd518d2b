"""Host-side check of a hardware rule that the compiler is trusted with, and that it once missed in a loop with a choice of paths.

An instruction other than a product that reads or overwrites the result of a matrix instruction has to stand some wait states behind it: this
compiler keeps 8 for the 16 x 16 products of bfloat16 and 10 for those of float32.  Where several paths through a loop's body met at its end,
copies of the accumulators came 2 to 7 behind the last product, and sums over more than one turn were wrong.  The delta rule's kernels, which
hold accumulators over loops, are compiled to ISA text (no GPU needed) and every way from a product to the first use of its result is followed.
Their loads from memory to LDS keep the rules for m0."""
import os
import re
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_isa_dpp_hazard import _functions

# result to any other instruction's operand, in wait states
NEEDED = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x4_f32": 10}
FILES = ["delta.hip", "delta_grad.hip"]


def _registers(token):
    token = token.strip().split(" ")[0].lstrip("-|").rstrip("|")
    one = re.match(r"([va])(\d+)$", token)
    if one:
        return {(one.group(1), int(one.group(2)))}
    some = re.match(r"([va])\[(\d+):(\d+)\]$", token)
    return {(some.group(1), i) for i in range(int(some.group(2)), int(some.group(3)) + 1)} if some else set()


def _parts(instruction):
    op, _, rest = instruction.partition(" ")
    return op, [x for x in re.split(r",(?![^\[]*\])", rest) if x]


def early_uses(text):
    """(function, product, use, wait states between) of every use that comes too early, and the number of products looked at"""
    early, products = [], 0
    for name, ins in _functions(text).items():
        labels = {l[:-1]: k for k, l in enumerate(ins) if l.endswith(":")}
        for k, product in enumerate(ins):
            op, args = _parts(product)
            if not op.startswith("v_mfma"):
                continue
            products += 1
            need = NEEDED[op]
            result = _registers(args[0])
            todo, seen = [(k + 1, 0)], {}
            while todo:
                j, waits = todo.pop()
                if j >= len(ins) or waits >= need or seen.get(j, need) <= waits:
                    continue
                seen[j] = waits
                if ins[j].endswith(":"):
                    todo.append((j + 1, waits))
                    continue
                op, args = _parts(ins[j])
                if op == "s_endpgm":
                    continue
                if op in ("s_branch",) or op.startswith("s_cbranch"):
                    todo.append((labels[args[0].strip()], waits + 1))
                    if op == "s_branch":
                        continue
                elif op.startswith("v_mfma"):
                    if (_registers(args[1]) | _registers(args[2])) & result:
                        early.append((name, product, ins[j], waits))
                        continue
                    if (_registers(args[0]) | _registers(args[3])) & result:
                        continue  # the next product of a sum: hardware passes the result on, and that product is looked at by itself
                elif op.startswith(("v_", "ds_", "global_", "scratch_", "buffer_", "flat_")):
                    if any(_registers(a) & result for a in args):
                        early.append((name, product, ins[j], waits))
                        continue
                todo.append((j + 1, waits + (int(args[0], 0) + 1 if op == "s_nop" else 1)))
    return early, products


_isa = {}


def _text(name):
    from paper_1710_08717_amd import build

    def one(name):
        with tempfile.TemporaryDirectory() as d:
            out = os.path.join(d, "out.s")
            r = subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", "-o", out, os.path.join(build.CSRC, name)],
                               capture_output=True, text=True)
            if r.returncode != 0:
                return None, r.stderr[-2000:]
            with open(out) as f:
                return f.read(), ""

    if not _isa:
        with ThreadPoolExecutor(max_workers=len(FILES)) as pool:
            _isa.update(zip(FILES, pool.map(one, FILES)))
    text, error = _isa[name]
    if text is None:
        pytest.fail("hipcc -S failed:\n" + error)
    return text


PRODUCT = " v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], v[0:3]\n"


@pytest.mark.parametrize("body,count", [
    (PRODUCT + " s_nop 6\n v_mov_b32_e32 v9, v2\n", 1),            # 7 where 8 are needed
    (PRODUCT + " s_nop 7\n v_mov_b32_e32 v9, v2\n", 0),
    (PRODUCT + " s_nop 6\n v_mov_b32_e32 v2, v9\n", 1),            # overwritten
    (PRODUCT + " s_nop 4\n ds_write_b128 v20, v[0:3]\n", 1),
    (PRODUCT + PRODUCT + " s_nop 7\n v_mov_b32_e32 v9, v2\n", 0),  # a sum of two products
    (PRODUCT + PRODUCT.replace("[8:11]", "[2:5]").replace("v[0:3]", "v[16:19]"), 1),  # a result as the next product's operand
    (PRODUCT + " s_cbranch_scc1 .LBB0_1\n s_nop 7\n.LBB0_1:\n v_mov_b32_e32 v9, v2\n", 1),  # one of two ways is too short
    (".LBB0_2:\n v_mov_b32_e32 v9, v2\n s_nop 7\n" + PRODUCT + " s_nop 2\n s_cbranch_scc1 .LBB0_2\n", 1),  # over a loop's end
])
def test_checker_sees_early_uses(body, count):
    early, products = early_uses("_Zk:\n" + body + " s_endpgm\n")
    assert len(early) == count and products >= 1


@pytest.mark.parametrize("name", FILES)
def test_results_of_products_are_waited_for(name):
    early, products = early_uses(_text(name))
    assert products >= 1000
    assert early == []


@pytest.mark.parametrize("name", FILES)
def test_loads_to_lds_set_m0_first(name):
    """and no instruction but such loads stands between: m0 is set, five wait states pass, up to four loads follow"""
    runs = 0
    for ins in _functions(_text(name)).values():
        for k, l in enumerate(ins):
            if not l.startswith("global_load_lds"):
                continue
            j = k
            while ins[j].startswith("global_load_lds"):
                j -= 1
            assert ins[j] == "s_nop 4" and ins[j - 1].startswith("s_mov_b32 m0,"), (ins[j - 1], ins[j], l)
            runs += 1
    assert runs >= 50
