"""The wait states around the matrix instructions that the weighted sum of drafted trees writes as asm statements in bf16, along every path through the built
code: branches are followed, and a product's accumulator is looked at as its operands are."""
import re

import pytest

import built_code
from test_tree_weighted_code import OPERAND, RESULT, WEIGHTED, _registers


def _instructions(text):
    """(address, name, arguments, address of a branch's target or None) of every instruction."""
    out = []
    for line in text.splitlines():
        code, _, note = line.partition("//")
        parts = code.replace(",", " ").split()
        where = re.match(r"\s*([0-9A-F]+)", note)
        if not parts or not where or not re.match(r"[a-z]+_", parts[0]):
            continue
        at = int(where[1], 16)
        target = None
        if "branch" in parts[0]:
            jump = int(parts[1], 0)
            target = at + 4 + 4 * (jump - 65536 if jump >= 32768 else jump)
        out.append((at, parts[0], parts[1:], target))
    return out


def _behind(name, args, early):
    """early: registers with the wait states that they still want, as an operand ("w") or at all ("r").  Returns (whether the instruction comes too
    early for one of them, the same behind it)."""
    regs = [_registers(t) for t in args]
    if name == "s_nop":
        return False, _later(early, int(args[0], 0) + 1)
    product = name.startswith("v_mfma")
    if product:
        out, a, b, c = regs[:4]
        wrong = any(("w", r) in early for r in a | b | c) or any(("r", r) in early for r in a | b | (c - out))
    else:
        wrong = any(("r", r) in early for some in regs for r in some)
    early = _later(early, 1)
    if product:
        early.update({("r", r): RESULT for r in out})
        for r in out:
            early.pop(("w", r), None)
    elif name.startswith("v_") and regs:
        for some in regs[:2] if "swap" in name else regs[:1]:
            early.update({("w", r): OPERAND for r in some})
    return wrong, early


def _later(early, states):
    return {k: n - states for k, n in early.items() if n > states}


def faults_of(text):
    """Instructions that come too early on some path, and how many products there are."""
    code = _instructions(text)
    index = {at: i for i, (at, *_) in enumerate(code)}
    state = {0: {}}
    todo, faults = [0], set()
    while todo:
        i = todo.pop()
        at, name, args, target = code[i]
        wrong, early = _behind(name, args, state[i])
        if wrong:
            faults.add(i)
        ways = []
        if target is not None:
            ways.append(index[target])
        if name not in ("s_branch", "s_endpgm") and i + 1 < len(code):
            ways.append(i + 1)
        for way in ways:
            old = state.get(way)
            new = dict(old or {})
            for k, n in early.items():
                new[k] = max(new.get(k, 0), n)
            if new != old:
                state[way] = new
                todo.append(way)
    return [code[i][:3] for i in sorted(faults)], sum(name.startswith("v_mfma") for _, name, *_ in code)


@pytest.mark.skipif(not built_code.PRESENT, reason="no disassembler")
@pytest.mark.parametrize("tiles", [1, 2, 3, 4, 6, 8])
def test_wait_states_on_every_path(tiles, tmp_path):
    faults, products = faults_of(built_code.disassembly(f"{WEIGHTED}Li{tiles}EEEvNS_8TreeArgsE", tmp_path))
    assert products >= 2 * 8 * tiles and not faults, faults[:5]


def _listing(*lines):
    return "\n".join(f"\t{line} // {4 * i:012X}: 00000000" for i, line in enumerate(lines))


def test_the_scan_finds_what_it_looks_for():
    product = "v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]"
    assert faults_of(_listing(product, product)) == ([], 2)
    assert len(faults_of(_listing("v_accvgpr_write_b32 a2, v9", "s_nop 0", product))[0]) == 1
    assert faults_of(_listing("v_accvgpr_write_b32 a2, v9", "s_nop 1", product)) == ([], 1)
    # a loop whose last instruction before the branch writes the first product's operand
    assert len(faults_of(_listing("s_nop 1", product, "v_mov_b32_e32 v1, v9", "s_cbranch_scc1 65533"))[0]) == 1
    assert faults_of(_listing("s_nop 1", product, "v_mov_b32_e32 v1, v9", "s_cbranch_scc1 65532")) == ([], 1)
    # read behind a branch over the wait
    late = ("s_cbranch_scc1 2", "s_nop 15", "s_nop 2", "v_accvgpr_read_b32 v9, a2")
    assert len(faults_of(_listing(product, *late))[0]) == 1
    assert faults_of(_listing(product, *late[1:])) == ([], 1)
