"""The matrix instructions of the product tiles are written out in the source, so the compiler neither knows how long they take nor
inserts the wait states behind them.  This checks the code that it generates: within the 20 wait states that a 32 x 32 x 64 instruction
may need, nothing but another such instruction that accumulates onto exactly the same registers reads or writes its result."""
import os
import re
import subprocess

import pytest

from paper_2512_22804_amd import build

WAIT_STATES = 20


def accumulators(operand):
    """AGPR numbers of an operand text such as a[16:31] or a7."""
    m = re.fullmatch(r"a\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.fullmatch(r"a(\d+)", operand)
    return {int(m.group(1))} if m else set()


def operands(text):
    return [o.strip() for o in text.split(",")]


def violations(lines):
    """(line, instruction) of every use of a result that is not there yet, in straight-line order; labels and branches only add time."""
    pending, bad = [], []               # (registers, wait states since)
    for number, line in enumerate(lines):
        line = line.split(";")[0].strip()
        m = re.match(r"([a-z][a-z0-9_]+)\s*(.*)", line)
        if not m or line.endswith(":"):
            continue
        name, ops = m.group(1), operands(re.sub(r"\s+(op_sel|cbsz|blgp|offset|offen|lds).*", "", m.group(2)))
        if name.startswith("s_nop"):
            states = int(ops[0], 0) + 1
        else:
            states = 1
            used = [accumulators(o) for o in ops]
            for registers, _ in pending:
                for k, u in enumerate(used):
                    if not u & registers:
                        continue
                    same = name.startswith("v_mfma") and k in (0, 3) and u == registers
                    if not same:
                        bad.append((number, line))
        pending = [(r, t + states) for r, t in pending if t + states < WAIT_STATES]
        if name.startswith("v_mfma"):
            pending.append((accumulators(ops[0]), 0))
    return bad


def test_checker():
    mfma = "v_mfma_scale_f32_32x32x64_f8f6f4 a[0:15], v[0:3], v[4:7], a[0:15], v8, v9 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
    assert violations([mfma, mfma]) == []
    assert violations([mfma, "v_accvgpr_read_b32 v1, a3"])
    assert violations([mfma, "v_accvgpr_mov_b32 a20, a15"])
    assert violations([mfma, "v_accvgpr_write_b32 a15, v2"])
    assert violations([mfma, mfma.replace("a[0:15]", "a[8:23]")])
    assert violations([mfma, "v_accvgpr_read_b32 v1, a16"]) == []
    assert violations([mfma, "s_nop 15", "s_nop 15", "v_accvgpr_read_b32 v1, a3"]) == []
    assert violations([mfma, "s_nop 7", "v_accvgpr_read_b32 v1, a3"])


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "mx_product.s"
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc, *[f for f in build.FLAGS if f != "-fPIC"], "-S", "--cuda-device-only", "-o", str(out),
                    os.path.join(build.CSRC, "mx_product.hip")], check=True, capture_output=True)
    found, name = {}, None
    for line in open(out):
        m = re.match(r"(_Z\w*k_mx_tile\w*):", line)
        if m:
            name = m.group(1)
            found[name] = []
        elif name:
            found[name].append(line)
            if "s_endpgm" in line and re.search(r"\.Lfunc_end", line):
                name = None
        if line.startswith(".Lfunc_end"):
            name = None
    return found


def test_nothing_touches_a_sum_too_early(kernels):
    assert len(kernels) == 12           # three modes, two result types, two tiles
    for name, lines in kernels.items():
        assert sum("v_mfma_scale_f32_32x32x64" in l for l in lines) >= 16
        assert violations(lines) == [], name


def test_sums_stay_in_registers(kernels):
    for name, lines in kernels.items():
        assert not any(re.match(r"\s*scratch_", l) for l in lines), name
