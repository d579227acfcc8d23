"""Loads from memory straight to LDS in the library's own kernels: the wait states that the hardware asks for.

The kernels issue these loads in inline assembly, where the compiler inserts none.  Of what a load reads, a scalar register that a
vector instruction wrote has to be 5 wait states before it, and an m0 that a scalar instruction wrote 1.  The instructions
before each load, on every way to it, are looked through in the built code.
"""
import concurrent.futures as cf
import os
import re
import shutil
import subprocess

import pytest

from paper_2407_10730_amd import build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
VECTOR_STATES, M0_STATES = 5, 1
KERNELS = {"softmax_prompt_kernel": 500, "softmax_step_kernel": 1000, "slice_conv_kernel": 50}  # loads that there are at least

_LOAD = re.compile(r"buffer_load_\w+ (.*) lds$")
# (of these the second operand is written too)
_TWO = re.compile(r"v_(add|sub|subrev|addc|subb|subbrev)_co|v_div_scale|v_mad_[iu]64")


def _scalars(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand) or re.fullmatch(r"s((\d+))", operand)
    return set(range(int(m[1]), int(m[2]) + 1)) if m else set()


def _operands(text):
    return [o.strip() for o in text.partition(" ")[2].split(",")]


def hazards(lines):
    """lines: a function's instructions and labels ("L1:").  Yields each load with what is written too shortly before it."""
    code, labels, branches = [], {}, {}
    for text in lines:
        if text.endswith(":"):
            labels.setdefault(len(code), []).append(text[:-1])
            continue
        m = re.match(r"s_c?branch\w* (\S+)", text)
        if m:
            branches.setdefault(m[1], []).append(len(code))
        code.append(text)
    for i, text in enumerate(code):
        m = _LOAD.match(text)
        if not m:
            continue
        reads = set().union(*(_scalars(o.split(" ")[0]) for o in _operands(text)))
        todo, seen = [(i, 0)], {}
        while todo:
            at, states = todo.pop()
            before = [b for label in labels.get(at, ()) for b in branches.get(label, ())]
            if at and not re.match(r"s_branch|s_endpgm|s_setpc", code[at - 1]):
                before.append(at - 1)
            for b in before:
                op = _operands(code[b])
                if code[b].startswith("v_") and states < VECTOR_STATES:
                    if reads & set().union(*map(_scalars, op[:2 if _TWO.match(code[b]) else 1])):
                        yield text, code[b], states
                if op[0] == "m0" and states < M0_STATES:
                    yield text, code[b], states
                m = re.match(r"s_nop (\d+)", code[b])
                more = states + (int(m[1]) + 1 if m else 1)
                if more < VECTOR_STATES and seen.get(b, 99) > more:
                    seen[b] = more
                    todo.append((b, more))


def _functions(path):
    """(name, lines) of the functions of a code object that load to LDS."""
    text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--symbolize-operands", path], capture_output=True, text=True,
                          check=True).stdout
    for part in re.split(r"^[0-9a-f]+ <(?=_Z)", text, flags=re.M)[1:]:
        name, _, body = part.partition(">:\n")
        if not re.search(r" lds\b", body):
            continue
        lines = []
        for line in body.splitlines():
            label = re.match(r"[0-9a-f]+ <(L\d+)>:", line)
            line = f"{label[1]}:" if label else re.sub(r"\s+", " ", line.partition("//")[0]).strip()
            if line:
                lines.append(line)
        yield name, lines


@pytest.fixture(scope="module")
def functions(tmp_path_factory):
    at = tmp_path_factory.mktemp("code")
    shutil.copy(build.LIB, at / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=at, capture_output=True, check=True)
    objects = [str(at / f) for f in os.listdir(at) if f.endswith("gfx950")]
    assert objects
    with cf.ThreadPoolExecutor(8) as ex:
        return [f for fs in ex.map(lambda p: list(_functions(p)), objects) for f in fs]


@pytest.mark.parametrize("kernel", KERNELS)
def test_loads_wait_for_what_they_read(functions, kernel):
    loads = 0
    for name, lines in functions:
        if kernel in name:
            loads += sum(bool(_LOAD.match(x)) for x in lines)
            assert not list(hazards(lines)), name
    assert loads >= KERNELS[kernel]


@pytest.mark.parametrize("before,bad", [
    (["v_readlane_b32 s2, v9, 3", "s_add_i32 m0, s8, 16", "s_nop 0"], True),
    (["v_readlane_b32 s2, v9, 3", "s_add_i32 m0, s8, 16", "s_nop 2"], True),
    (["v_readlane_b32 s2, v9, 3", "s_add_i32 m0, s8, 16", "s_nop 3"], False),
    (["v_readlane_b32 s4, v9, 3", "s_add_i32 m0, s8, 16", "s_nop 0"], False),
    (["v_cmp_eq_u32_e64 s[0:1], v9, 3", "s_mov_b32 m0, s8", "s_nop 0"], True),
    (["s_nop 7", "s_mov_b32 m0, s8"], True),
    (["v_readfirstlane_b32 s0, v1", "s_branch L1", "L0:", "s_nop 7", "L1:", "s_mov_b32 m0, s8", "s_nop 0"], True),
    (["v_readfirstlane_b32 s0, v1", "s_branch L2", "L1:", "s_mov_b32 m0, s8", "s_nop 0"], False),
])
def test_what_counts_as_too_shortly_before(before, bad):
    assert bool(list(hazards(before + ["buffer_load_dwordx4 v7, s[0:3], 0 offen lds"]))) == bad
