"""Waits that the instructions of the products need and that the compiler cannot see to, in its own assembly of them (no GPU)."""
import os
import re
import subprocess

import pytest

from paper_1503_05032_amd import build as libbuild


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel: its instructions and labels} of grouped.hip, by the flags of the library."""
    out = str(tmp_path_factory.mktemp("waits") / "grouped.s")
    source = next(s for s in libbuild.SRC if s.endswith("grouped.hip"))
    subprocess.run([libbuild.hipcc(), *libbuild.FLAGS, "-I", libbuild.INC, "-S", "--cuda-device-only", source, "-o", out], check=True, stdin=subprocess.DEVNULL,
                   stderr=subprocess.DEVNULL)
    found, name = {}, None
    with open(out) as f:
        for line in f:
            text = line.split(";")[0].split("//")[0].strip()
            start = re.match(r"(_ZN\S*k_product\S*):$", text)
            if start:
                name = start[1]
                found[name] = []
            elif text.startswith(".Lfunc_end"):
                name = None
            elif name and text and (text.endswith(":") or not text.startswith(".")):
                found[name].append(text)
    assert len(found) > 50
    return found


def test_loads_into_lds_have_their_base_from_a_scalar_instruction(kernels):
    """Right before each: five states would be needed after a vector one; and m0 one state before, by a scalar one too."""
    loads = 0
    for name, code in kernels.items():
        for i, text in enumerate(code):
            load = re.match(r"global_load_lds_\w+ v\S+, (\S+)", text)
            if not load:
                continue
            loads += 1
            assert code[i - 2].startswith("s_mov_b32 m0, s"), (name, code[i - 2:i + 1])
            if load[1] == "off":
                assert code[i - 1] == "s_nop 0", (name, code[i - 2:i + 1])
            else:
                assert code[i - 1].startswith(f"s_mov_b64 {load[1]}, s["), (name, code[i - 2:i + 1])
    assert loads > 1000


# Wait states until the results of a matrix instruction may be read or written by anything but another one: of 8 passes 12, of 4
# passes 8.
STATES = {"v_mfma_f32_16x16x128_f8f6f4": 12, "v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x32_f16": 8}


def registers(operands):
    """Vector and accumulation registers that are named there."""
    out = set()
    for kind, first, last, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", operands):
        out.update((kind, i) for i in (range(int(first), int(last) + 1) if first else (int(one),)))
    return out


def touched_early(code):
    """Matrix instructions whose results something touches too early on some path through the kernel, and with what; how many
    matrix instructions there are."""
    label = {text[:-1]: i for i, text in enumerate(code) if text.endswith(":")}
    named = [set() if text.endswith(":") else registers(text.partition(" ")[2]) for text in code]

    def following(i):
        branch = re.match(r"s_c?branch\S*\s+(\S+)", code[i])
        if branch:
            yield label[branch[1]]
        if not code[i].startswith(("s_branch", "s_endpgm")):
            yield i + 1

    early, count = [], 0
    for i, text in enumerate(code):
        if not text.startswith("v_mfma"):
            continue
        count += 1
        op, operands = text.split(None, 1)
        results, seen, paths = registers(operands.split(",")[0]), {}, [(j, 0) for j in following(i)]
        while paths:
            j, states = paths.pop()
            if states >= STATES[op] or seen.get(j, 99) <= states:
                continue
            seen[j] = states
            if not code[j].startswith("v_mfma") and named[j] & results:
                early.append((text, code[j], states))
                continue
            nop = re.match(r"s_nop (\d+)", code[j])
            states += 0 if code[j].endswith(":") else int(nop[1]) + 1 if nop else 1
            paths += [(k, states) for k in following(j)]
    return early, count


def test_results_of_matrix_instructions_are_not_touched_too_early(kernels):
    """A branch around what reads such a result once led to a write of its registers that the instruction's own came after."""
    total = 0
    for name, code in kernels.items():
        early, count = touched_early(code)
        assert not early, (name, early)
        assert count > 0, name
        total += count
    assert total > 2000


def test_an_early_touch_is_seen():
    product = "v_mfma_f32_16x16x32_bf16 v[4:7], v[8:11], v[12:15], 0"
    assert touched_early([product, "s_nop 6", "v_mul_f32_e32 v1, v2, v5", "s_endpgm"])[0] == [(product, "v_mul_f32_e32 v1, v2, v5", 7)]
    assert touched_early([product, "s_nop 7", "v_mul_f32_e32 v1, v2, v5", "s_endpgm"]) == ([], 1)
    around = [product, "s_cbranch_scc1 .L1", "s_nop 7", "v_add_f32_e32 v1, v4, v4", ".L1:", "v_mov_b32_e32 v7, 0", "s_endpgm"]
    assert touched_early(around)[0] == [(product, "v_mov_b32_e32 v7, 0", 1)]
    loop = [".L0:", "v_mov_b32_e32 v3, v6", "s_nop 1", product, "s_cbranch_scc0 .L0", "s_endpgm"]
    assert touched_early(loop)[0] == [(product, "v_mov_b32_e32 v3, v6", 1)]
    held = ["v_accvgpr_read_b32 v0, a3", "s_endpgm"]
    assert touched_early([product.replace("v[4:7]", "a[0:3]"), *held])[0]
