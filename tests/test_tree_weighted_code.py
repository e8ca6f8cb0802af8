"""The wait states around the matrix instructions that the weighted sum of drafted trees writes as asm statements in bf16, of which the compiler knows
nothing: read from the built library, instruction after instruction."""
import re

import pytest

import built_code

WEIGHTED = "_ZN4slim12_GLOBAL__N_120tree_weighted_kernelILi1E"
OPERAND, RESULT = 2, 19            # wait states: vector write -> operand of a product; product -> any other use of its accumulator (16 passes and 3)


def _registers(token):
    m = re.fullmatch(r"([av])\[(\d+):(\d+)\]", token)
    if m:
        return {(m[1], i) for i in range(int(m[2]), int(m[3]) + 1)}
    m = re.fullmatch(r"([av])(\d+)", token)
    return {(m[1], int(m[2]))} if m else set()


def _faults(text):
    """Instructions that come too early, and how many products there are."""
    faults, products, now, ready, written = [], 0, 0, {}, {}
    for line in text.splitlines():
        parts = line.split("//")[0].replace(",", " ").split()
        if not parts or not re.match(r"[a-z]+_", parts[0]):
            continue
        name, args = parts[0], [_registers(t) for t in parts[1:]]
        if name == "s_nop":
            now += int(parts[1], 0) + 1
            continue
        if name.startswith("v_mfma"):
            products += 1
            out, a, b, c = args[:4]
            early = any(now - written.get(r, -OPERAND - 1) - 1 < OPERAND for r in a | b) or any(now < ready.get(r, 0) for r in a | b | (c - out))
            ready.update({r: now + 1 + RESULT for r in out})
        else:
            early = any(now < ready.get(r, 0) for regs in args for r in regs)
            if name.startswith("v_") and args:
                written.update({r: now for r in args[0]})
        if early:
            faults.append(line.strip())
        now += 1
    return faults, products


@pytest.mark.skipif(not built_code.PRESENT, reason="no disassembler")
@pytest.mark.parametrize("tiles", [1, 2, 3, 4, 6, 8])
def test_wait_states(tiles, tmp_path):
    faults, products = _faults(built_code.disassembly(f"{WEIGHTED}Li{tiles}EEEvNS_8TreeArgsE", tmp_path))
    assert products >= 2 * 8 * tiles and not faults, faults[:5]


def test_the_scan_finds_what_it_looks_for():
    product = "v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]\n"
    assert _faults(product * 2) == ([], 2)
    assert _faults("v_mov_b32_e32 v1, v9\ns_nop 1\n" + product) == ([], 1)
    assert len(_faults("v_mov_b32_e32 v1, v9\ns_nop 0\n" + product)[0]) == 1
    assert len(_faults(product + "s_nop 15\nv_accvgpr_read_b32 v9, a2\n")[0]) == 1
    assert _faults(product + "s_nop 15\ns_nop 2\nv_accvgpr_read_b32 v9, a2\n") == ([], 1)
