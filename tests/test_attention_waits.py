"""Waits that the attention's instructions need: its loads into LDS, whose assembly the compiler does not look into, and its matrix instructions'
results along every path of the compiled kernels (no GPU)."""
import re
import subprocess

import pytest

import test_kernel_waits as waits
from paper_1503_05032_amd import build as libbuild

# As in test_kernel_waits: wait states until results may be touched, of instructions of 8 passes.
STATES = {"v_mfma_f32_32x32x16_bf16": 12, "v_mfma_f32_32x32x16_f16": 12}


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel: its instructions and labels} of the attention's sources, by the flags of the library, compiled side by side."""
    folder = tmp_path_factory.mktemp("waits")
    sources = [s for s in libbuild.SRC if s.endswith(("attention.hip", "attention_back.hip"))]
    assert len(sources) == 2
    outs = [str(folder / f"{i}.s") for i in range(2)]
    running = [subprocess.Popen([libbuild.hipcc(), *libbuild.FLAGS, "-I", libbuild.INC, "-S", "--cuda-device-only", source, "-o", out], stdin=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
               for source, out in zip(sources, outs)]
    assert [p.wait() for p in running] == [0, 0]
    found, name = {}, None
    for out in outs:
        with open(out) as f:
            for line in f:
                text = line.split(";")[0].split("//")[0].strip()
                start = re.match(r"(_ZN\S*k_attend\S*):$", text)
                if start:
                    name = start[1]
                    found[name] = []
                elif text.startswith(".Lfunc_end"):
                    name = None
                elif name and text and (text.endswith(":") or not text.startswith(".")):
                    found[name].append(text)
    assert len(found) > 100
    return found


def test_loads_into_lds_have_their_base_from_a_scalar_instruction(kernels):
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


def test_results_of_matrix_instructions_are_not_touched_too_early(kernels, monkeypatch):
    monkeypatch.setattr(waits, "STATES", waits.STATES | STATES)
    total = 0
    for name, code in kernels.items():
        early, count = waits.touched_early(code)
        assert not early, (name, early)
        assert count > 0, name
        total += count
    assert total > 2000
