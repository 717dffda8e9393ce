"""Listings of the kernels that use matrix instructions: on no path is a result read, or its registers written again, before it is there.

The hardware does not hold back an instruction that reads the result of a matrix instruction too early; the compiler has to put instructions or s_nop between
them, also where the path goes through branches and round loops.  A missing one gives wrong numbers that need not show in another test."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_1905_12799_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# Instructions that have to lie between a result and its use (s_nop n counts n + 1): what the compiler keeps between two that follow each other directly.  A write
# of the same registers may come one earlier.
WAITS = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x4_f32": 10, "v_mfma_f32_32x32x16_f16": 12, "v_mfma_f32_32x32x16_bf16": 12}


def registers(operand):
    m = re.match(r"[-|]*[va](?:(\d+)|\[(\d+):(\d+)\])", operand)
    if not m:
        return set()
    return {int(m[1])} if m[1] else set(range(int(m[2]), int(m[3]) + 1))


def functions(listing):
    """(name, instructions as (opcode, operands, text), where labels are) of every kernel."""
    for name, body in re.findall(r"^(_Z\w+):.*?\n(.*?)\.Lfunc_end", listing, re.S | re.M):
        code, labels = [], {}
        for line in body.split("\n"):
            line = line.split(";")[0].strip()
            if re.match(r"[.$\w]+:$", line):
                labels[line[:-1]] = len(code)
            elif line and not line.startswith("."):
                op, *rest = line.split(None, 1)
                code.append((op, [x.strip() for x in rest[0].split(",")] if rest else [], line))
        yield name, code, labels


def too_early(op, result, waited, other, operands):
    """Whether `other`, so many instructions behind, takes or overwrites the result before it is there; None where it does neither."""
    need = WAITS[op]
    if other.startswith("v_mfma"):
        c, d = registers(operands[3]), registers(operands[0])
        if (registers(operands[1]) | registers(operands[2])) & result:
            return waited < need
        if c == result and WAITS[other] == WAITS[op]:    # (handed on inside the matrix unit)
            return False
        return waited < need if (c | d) & result else None
    if other[0] not in "vdgb":                           # vector, LDS, global, buffer
        return None
    stores = "store" in other or "write" in other or other.startswith("v_cmp")
    reads = set().union(*(registers(x) for x in (operands if stores else operands[1:])))
    if reads & result:
        return waited < need
    return waited < need - 1 if operands and registers(operands[0]) & result else None


def early_uses(listing):
    found, matrix = [], 0
    for name, code, labels in functions(listing):
        for i, (op, operands, text) in enumerate(code):
            if not op.startswith("v_mfma"):
                continue
            matrix += 1
            assert op in WAITS, f"{op}: how long its result takes is not in the table"
            result, seen, paths = registers(operands[0]), {}, [(i + 1, 0)]
            while paths:
                at, waited = paths.pop()
                while at < len(code) and waited < WAITS[op] and seen.get(at, 99) > waited:
                    seen[at] = waited
                    other, others, line = code[at]
                    early = too_early(op, result, waited, other, others)
                    if early:
                        found.append(f"{name}: {text} | {waited} between | {line}")
                    if early is not None or other == "s_endpgm":
                        break
                    waited += int(others[0], 0) + 1 if other == "s_nop" else 1
                    if other == "s_branch":
                        at = labels[others[0]]
                        continue
                    if other.startswith("s_cbranch"):
                        paths.append((labels[others[0]], waited))
                    at += 1
    return found, matrix


def kernel(*lines):
    return "_Zkernel:\n" + "\n".join("\t" + x if not x.endswith(":") else x for x in lines) + "\n\ts_endpgm\n.Lfunc_end0:\n"


PRODUCT = "v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], 0"


def test_what_is_found():
    read = "v_add_f32_e32 v20, v1, v21"
    for lines, early in (([PRODUCT, read], 1), ([PRODUCT, "s_nop 7", read], 0), ([PRODUCT, "s_nop 6", read], 1),
                         ([PRODUCT, "s_nop 6", "v_mov_b32_e32 v2, 0"], 0), ([PRODUCT, "s_nop 5", "v_mov_b32_e32 v2, 0"], 1),
                         ([PRODUCT, "global_store_dwordx4 v[30:31], v[0:3], off"], 1), ([PRODUCT, "ds_write_b128 v30, v[0:3]"], 1),
                         # handed on as it is, or as an operand
                         ([PRODUCT, "v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], v[0:3]", "s_nop 7", read], 0),
                         ([PRODUCT, "v_mfma_f32_16x16x32_bf16 v[4:7], v[0:3], v[12:15], 0"], 1),
                         # past a branch, on the way that is taken and on the one that is not, and round a loop
                         ([PRODUCT, "s_cbranch_scc1 .L1", "s_nop 7", ".L1:", read], 1), ([PRODUCT, "s_cbranch_scc1 .L1", read, ".L1:"], 1),
                         ([PRODUCT, "s_branch .L1", read, ".L1:", "s_nop 7", read], 0), ([".L1:", read, "s_nop 7", PRODUCT, "s_cbranch_scc0 .L1"], 1),
                         ([".L1:", "s_nop 7", read, PRODUCT, "s_cbranch_scc0 .L1"], 0)):
        found, matrix = early_uses(kernel(*lines))
        assert bool(found) == bool(early) and matrix >= 1, (lines, found)


def test_no_result_is_used_too_early():
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")

    def uses(name):
        done = subprocess.run([HIPCC, *build.compile_flags(), "--cuda-device-only", "-S", "-o", "-", os.path.join(build.CSRC, name)], capture_output=True, text=True)
        assert done.returncode == 0, done.stderr
        return early_uses(done.stdout)
    units = ["gated_delta.hip", "kmeans_lloyd.hip", "kmeans_small.hip", "matrix_step.hip"]       # (of the Lloyd step, what is built for up to 8 features)
    for source in build.sources():
        with open(source) as f:
            assert "__builtin_amdgcn_mfma" not in f.read() or os.path.basename(source) in units, source
    with ThreadPoolExecutor(len(units)) as pool:
        for unit, (found, matrix) in zip(units, pool.map(uses, units)):
            assert matrix > 0 and not found, (unit, found[:5])
