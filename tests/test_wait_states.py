"""The built library's own gfx950 code: wait states that the hardware leaves to the program.

A vector instruction that writes a scalar register (v_readfirstlane, v_readlane, comparisons, carries) has to be five wait states ahead of a memory instruction that
reads the register, and a write of m0 one ahead of a load to LDS.  The compiler sees to that for its own instructions; what inline assembly contains it does not look at.  Every instruction is one
wait state, s_nop n is n + 1.  Followed through branches inside a function; calls and returns begin anew.
"""
import os
import re
import shutil
import subprocess

import pytest

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
VALU_TO_MEMORY, M0_TO_LDS = 5, 1
LINE = re.compile(r"^\s+([a-z]\w*)\s*(.*?)\s*// ([0-9A-F]{12}):(.*)$")
TARGET = re.compile(r"<[^>]*?\+0x([0-9a-f]+)>|<[^>+]+>\s*$")
SCALAR = re.compile(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b|\b(vcc)(?:_lo|_hi)?\b|\b(m0)\b")
MEMORY = ("buffer_", "global_", "flat_", "scratch_")
TWO_RESULTS = ("v_add_co", "v_sub_co", "v_subrev_co", "v_addc_co", "v_subb_co", "v_subbrev_co", "v_div_scale", "v_mad_u64", "v_mad_i64")


def scalars(text):
    found = set()
    for m in SCALAR.finditer(text):
        if m.group(1):
            found.update(range(int(m.group(1)), int(m.group(2)) + 1))
        elif m.group(3):
            found.add(int(m.group(3)))
        else:
            found.add(m.group(4) or m.group(5))
    return found


def operands(text):
    return [p.strip() for p in text.split(", ")]


def too_soon(instructions, start):
    """(address, instruction, register) of every read that comes too soon.  instructions: (address, name, operands, target) in order."""
    waiting, bad, arriving = {}, set(), {}

    def merge(into, other):
        changed = False
        for r, d in other.items():
            if d < into.get(r, 99):
                into[r] = d
                changed = True
        return changed
    again, rounds = True, 0
    while again and rounds < 8:
        again, rounds, waiting = False, rounds + 1, {}
        for address, name, text, target in instructions:
            if address in arriving:
                merge(waiting, arriving[address])
            # waiting[register]: wait states since it was written
            if waiting and name.startswith(MEMORY):
                for r in scalars(text) & waiting.keys():
                    if r != "m0" and waiting[r] < VALU_TO_MEMORY:
                        bad.add((address, name + " " + text, "s%s" % r))
                if text.endswith(" lds") or "_lds_" in name:
                    if waiting.get("m0", 99) < M0_TO_LDS:
                        bad.add((address, name + " " + text, "m0"))
            states = int(text) + 1 if name == "s_nop" else 1
            if waiting:
                waiting = {r: d + states for r, d in waiting.items() if d + states < (M0_TO_LDS if r == "m0" else VALU_TO_MEMORY)}
            if name.startswith("v_"):
                parts = operands(text)
                if name.startswith("v_cmpx"):
                    parts = []
                for p in parts[:2] if name.startswith(TWO_RESULTS) else parts[:1]:
                    if p[:1] == "s" or p[:3] == "vcc":
                        for r in scalars(p):
                            waiting[r] = 0
            elif name.startswith("s_"):
                if target is not None and waiting:
                    if merge(arriving.setdefault(target, {}), waiting):
                        again = True
                if name in ("s_branch", "s_endpgm", "s_setpc_b64", "s_swappc_b64"):
                    waiting = {}
                elif text.startswith("m0"):
                    waiting["m0"] = 0
    return bad


def functions(code_object):
    text = subprocess.run([OBJDUMP, "-d", code_object], stdout=subprocess.PIPE, check=True, text=True).stdout
    name, start, body = None, 0, []
    for line in text.splitlines():
        m = LINE.match(line)
        if m:
            target = None
            if m.group(1).startswith(("s_cbranch", "s_branch")):
                t = TARGET.search(m.group(4))
                target = start + int(t.group(1) or "0", 16) if t else None
            body.append((int(m.group(3), 16), m.group(1), m.group(2), target))
        elif line.endswith(">:"):
            if body:
                yield name, start, body
            start, name, body = int(line.split()[0], 16), line.split("<")[1][:-2], []
    if body:
        yield name, start, body


@pytest.fixture(scope="module")
def code_objects(tmp_path_factory):
    from paper_2601_16536_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    folder = tmp_path_factory.mktemp("code")
    shutil.copy(binding.LIB_PATH, str(folder / "lib.so"))
    subprocess.check_call([OBJDUMP, "--offloading", "lib.so"], cwd=str(folder), stdout=subprocess.DEVNULL)
    return sorted(str(folder / f) for f in os.listdir(str(folder)) if f.endswith("gfx950"))


def test_the_check_sees_what_it_is_for():
    """A bound that a vector instruction writes two states ahead of its load, the same five ahead, and over a branch back."""
    load = (100, "buffer_load_dwordx4", "v1, s[4:7], 0 offen lds", None)
    first = (80, "v_readfirstlane_b32", "s6, v0", None)
    m0 = [(84, "s_mov_b32", "m0, s9", None), (88, "s_nop", "0", None)]
    assert too_soon([first] + m0 + [load], 80) == {(100, "buffer_load_dwordx4 v1, s[4:7], 0 offen lds", "s6")}
    assert not too_soon([first, m0[0], (88, "s_nop", "3", None), load], 80)
    assert {r for _, _, r in too_soon([first, (84, "s_mov_b32", "m0, s9", None), load], 80)} == {"s6", "m0"}
    assert not too_soon([(80, "v_cmp_eq_u32_e64", "s[8:9], v0, v1", None)] + m0 + [load], 80)
    assert {r for _, _, r in too_soon([m0[0], (88, "s_nop", "0", None), load, first, (108, "s_cbranch_scc1", "x", 84), (112, "s_endpgm", "", None)], 84)} == {"s6"}


@pytest.fixture(scope="module")
def checked(code_objects):
    """Of all functions: how many memory instructions, the reads that come too soon, calls."""
    seen, soon, calls = 0, [], []
    for path in code_objects:
        for name, start, body in functions(path):
            seen += sum(1 for i in body if i[1].startswith(MEMORY))
            soon += [(name, "%x" % a, i, r) for a, i, r in sorted(too_soon(body, start))]
            calls += [name for i in body if i[1] in ("s_swappc_b64", "s_call_b64")]
    return seen, soon, calls


def test_scalar_operands_are_there_in_time(checked):
    seen, soon, _ = checked
    assert seen > 10000
    assert not soon, "%d reads too soon, the first %r" % (len(soon), soon[:12])


def test_loops_call_no_function(checked):
    """A function of its own gets what it needs through scratch memory, and waits there for the loads that a loop has on their way."""
    assert not checked[2], sorted(set(checked[2]))
