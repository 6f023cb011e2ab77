"""The loads that the matrix products write in assembly, in the code that the compiler makes around them: a vector memory instruction
must not read a scalar register fewer than five wait states after a vector instruction wrote it, and the compiler, which sees to
that elsewhere, does not look into assembly.  Nor may anything else rely on m0, which those loads set."""
import re
import subprocess

import pytest

from paper_1901_01544_amd import build


def scalar_registers(operand):
    found = {int(n) for n in re.findall(r"(?<![\w\[:])s(\d+)\b", operand)}
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", operand):
        found |= set(range(int(a), int(b) + 1))
    return found


def written_by_vector(line):
    """Scalar registers that a vector instruction writes."""
    if not line.startswith("v_"):
        return set()
    operands = line.split(None, 1)[1].split(",")
    two = re.match(r"v_(add|sub|subrev|addc|subb|subbrev)c?_co|v_div_scale|v_mad_u64", line)
    return scalar_registers(operands[0]) | (scalar_registers(operands[1]) if two else set())


def too_close(lines, want=5):
    """(loads, [(load, writer), ...]): along every path of control flow."""
    label = {l[:-1]: i for i, l in enumerate(lines) if l.startswith(".LBB")}
    jumps = {}
    for i, l in enumerate(lines):
        m = re.match(r"s_c?branch\w*\s+(\.LBB\w+)", l)
        if m:
            jumps.setdefault(label[m[1]], []).append(i)

    def before(i):
        falls = i > 0 and not lines[i - 1].startswith(("s_branch", "s_endpgm"))
        return jumps.get(i, []) + ([i - 1] if falls else [])

    loads, found = 0, []
    for i, l in enumerate(lines):
        if not l.startswith("global_load_lds"):
            continue
        loads += 1
        base, seen, todo = scalar_registers(l.split(",")[-1]), set(), [(j, 0) for j in before(i)]
        while todo:
            j, waited = todo.pop()
            if waited >= want or (j, waited) in seen:
                continue
            seen.add((j, waited))
            p = lines[j]
            if p.startswith(".LBB"):
                todo += [(k, waited) for k in before(j)]
                continue
            if written_by_vector(p) & base:
                found.append((l, p))
            states = int(p.split()[1], 0) + 1 if p.startswith("s_nop") else 1
            todo += [(k, waited + states) for k in before(j)]
    return loads, found


def code(text):
    lines = [l.split(";")[0].strip() for l in text.splitlines()]
    return [l for l in lines if l and (not l.startswith(".") or re.match(r"\.LBB\w+:", l))]


def test_the_search_finds_what_it_looks_for():
    close = "a:\nv_readfirstlane_b32 s4, v1\ns_mov_b32 m0, s9\ns_nop 0\nglobal_load_lds_dwordx4 v0, s[4:5]\n"
    assert too_close(code(close)) == (1, [("global_load_lds_dwordx4 v0, s[4:5]", "v_readfirstlane_b32 s4, v1")])
    assert too_close(code(close.replace("s_nop 0", "s_nop 4"))) == (1, [])
    assert too_close(code(close.replace("s4, v1", "s6, v1"))) == (1, [])
    round_a_loop = ".LBB0_1:\nglobal_load_lds_dwordx4 v0, s[4:5]\ns_add_u32 s8, s8, 1\nv_cmp_eq_u32_e64 s[4:5], v0, v1\ns_cbranch_scc1 .LBB0_1\n"
    assert len(too_close(code(round_a_loop))[1]) == 1


def test_waits_around_the_loads(tmp_path):
    source = next(s for s in build.SOURCES if s.endswith("iwp_losses.hip"))
    out = str(tmp_path / "losses.s")
    done = subprocess.run([build.hipcc(), *build.HIPCC_FLAGS, "--cuda-device-only", "-S", "-o", out, source], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr[-2000:]
    text = open(out).read()
    loads = 0
    for function in re.split(r"\n(?=_ZN3iwp\w+:)", text)[1:]:
        lines = code(function.split(".Lfunc_end")[0])
        n, found = too_close(lines)
        assert not found, found[:3]
        loads += n
        assert all(l.startswith("s_mov_b32 m0,") for l in lines if re.search(r"\bm0\b", l))
    assert loads > 100
