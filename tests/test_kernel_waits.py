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
