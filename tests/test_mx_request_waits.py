"""The product tiles' requests into LDS are written out in the source too.  Each reads its buffer resource from scalar registers, and the
compiler, which does not look into the text, does not keep the five wait states that must lie between a vector instruction that writes
a scalar register (v_readfirstlane, v_readlane) and a buffer load that reads it.  So the text has to hold them itself, whatever
stands before it.  The check of the sums is repeated here along every way that the program can take, loops included."""
import re

from test_mx_wait_states import WAIT_STATES, accumulators, kernels, operands  # noqa: F401 (a fixture)

REQUEST_STATES = 5


def states_of(line):
    name, _, rest = line.partition(" ")
    return int(rest.split(",")[0], 0) + 1 if name == "s_nop" else 1


def requests(lines):
    """(line, wait states in its own text before it) of every written-out buffer load."""
    found, inside = [], None
    for number, line in enumerate(lines):
        if ";#ASMSTART" in line:
            inside = 0
        elif ";#ASMEND" in line:
            inside = None
        elif inside is not None:
            text = line.split(";")[0].strip()
            if text.startswith("buffer_load"):
                found.append((number, inside))
            if text:
                inside += states_of(re.sub(r"\s+", " ", text))
    return found


def program(lines):
    """Instructions as (line, name, operands), and the place of every label."""
    code, labels = [], {}
    for number, line in enumerate(lines):
        text = line.split(";")[0].strip()
        m = re.match(r"(\.L\w+):", text)
        if m:
            labels[m.group(1)] = len(code)
            continue
        m = re.match(r"([a-z][a-z0-9_]+)\s*(.*)", text)
        if m:
            code.append((number, m.group(1), operands(re.sub(r"\s+(op_sel|cbsz|blgp|offset|offen|lds).*", "", m.group(2)))))
    return code, labels


def early_uses(lines):
    """Lines that read or write a matrix instruction's result before it is there, on any way from it."""
    code, labels = program(lines)
    bad = set()
    for start, (_, name, ops) in enumerate(code):
        if not name.startswith("v_mfma"):
            continue
        registers, least, ways = accumulators(ops[0]), {}, [(start + 1, 0)]
        while ways:
            at, since = ways.pop()
            if at >= len(code) or since >= WAIT_STATES or least.get(at, WAIT_STATES) <= since:
                continue
            least[at] = since
            number, other, used = code[at]
            if other == "s_endpgm":
                continue
            for k, operand in enumerate(used):
                u = accumulators(operand)
                if u & registers and not (other.startswith("v_mfma") and k in (0, 3) and u == registers):
                    bad.add(number)
            after = since + (int(used[0], 0) + 1 if other == "s_nop" else 1)
            if other.startswith(("s_branch", "s_cbranch")):
                ways.append((labels[used[0]], after))
            if other != "s_branch":
                ways.append((at + 1, after))
    return sorted(bad)


MFMA = "v_mfma_scale_f32_32x32x64_f8f6f4 a[0:15], v[0:3], v[4:7], a[0:15], v8, v9 op_sel_hi:[0,0,0] cbsz:4 blgp:4"


def test_checkers():
    asm = lambda nop: [";#ASMSTART", "s_mov_b32 m0, s1", f"s_nop {nop}", "buffer_load_dwordx4 v1, s[0:3], 0 offen lds", ";#ASMEND"]
    assert requests(asm(0)) == [(3, 2)] and requests(asm(3)) == [(3, 5)]
    assert requests(["buffer_load_dwordx4 v1, s[0:3], 0 offen"]) == []          # the compiler's own
    loop = [".LBB0_1:", "v_accvgpr_read_b32 v1, a3", "s_nop 15", "s_nop 15", MFMA, "s_cbranch_scc1 .LBB0_1", "s_endpgm"]
    assert early_uses(loop) == [1]
    assert early_uses([loop[0], *loop[2:4], loop[1], *loop[4:]]) == []
    assert early_uses([MFMA, "s_branch .LBB0_2", "v_accvgpr_read_b32 v1, a3", ".LBB0_2:", "s_endpgm"]) == []
    assert early_uses([MFMA, MFMA, "s_endpgm"]) == []


def test_requests_keep_their_distance(kernels):  # noqa: F811
    for name, lines in kernels.items():
        found = requests(lines)
        assert len(found) >= 16, name
        assert all(states >= REQUEST_STATES for _, states in found), f"{name}: {min(s for _, s in found)} wait states"


def test_nothing_touches_a_sum_too_early_on_any_way(kernels):  # noqa: F811
    for name, lines in kernels.items():
        assert early_uses(lines) == [], name
