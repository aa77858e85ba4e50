"""The loads straight into LDS are written in assembly, where the compiler adds
no wait states. CDNA3 and CDNA4 want five between a vector instruction that
writes a scalar register (v_readfirstlane_b32) and a memory instruction that
reads it, and one between a write of m0 and a load to LDS. Compiled here for the
worst caller, whose base is a lane's value read right before the load."""
import os
import re
import subprocess

import pytest

from paper_2306_10015_amd import build

SOURCE = r'''
#include "lds_dma.hpp"
__global__ void probe(const uint64_t* base, const uint32_t* offset, uint32_t* out)
{
    __shared__ uint32_t lds[256];
    const uint64_t at = base[threadIdx.x];
    const uint32_t off = offset[threadIdx.x];
    const uint64_t first = uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at >> 32)))) << 32 |
                           uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at)));
    LOAD(first, off, mezo::lds_offset(lds));
    mezo::dma_wait();
    out[threadIdx.x] = lds[threadIdx.x];
}
'''


def registers(text):
    """The scalar registers that an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", text)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.fullmatch(r"s(\d+)", text)
    return {int(m.group(1))} if m else set()


def states(instruction):
    m = re.match(r"s_nop (\d+)", instruction)
    return int(m.group(1)) + 1 if m else 1


def missing_waits(instructions):
    """(load, what it does not wait for) of each load to LDS."""
    bad = []
    for i, load in enumerate(instructions):
        m = re.match(r"global_load_lds_dword\w* [^,]+, (\S+)", load)
        if not m:
            continue
        open_registers, passed = registers(m.group(1)), 0
        for before in reversed(instructions[:i]):
            if passed == 0 and re.match(r"s_mov_b32 m0,", before):
                bad.append((load, before))
            w = re.match(r"([sv]_\w+) (s\[\d+:\d+\]|s\d+|m0)", before)
            if w:
                written = registers(w.group(2)) & open_registers
                if written and w.group(1).startswith("v_") and passed < 5:
                    bad.append((load, before))
                open_registers = open_registers - written
            passed += states(before)
            if passed >= 5:
                break
    return bad


def test_the_check_itself():
    assert missing_waits(["v_readfirstlane_b32 s4, v1", "s_mov_b32 m0, s2", "s_nop 0",
                          "global_load_lds_dwordx4 v0, s[4:5]"])
    assert missing_waits(["s_mov_b32 m0, s2", "global_load_lds_dword v0, s[4:5]"])
    assert not missing_waits(["v_readfirstlane_b32 s4, v1", "s_mov_b32 m0, s2", "s_nop 3",
                              "global_load_lds_dwordx4 v0, s[4:5]"])
    assert not missing_waits(["v_readfirstlane_b32 s4, v1", "s_mov_b32 m0, s2", "s_mov_b64 s[6:7], s[4:5]",
                              "global_load_lds_dwordx4 v0, s[6:7]"])


@pytest.mark.parametrize("load", ["dma_to_lds", "dma_word_to_lds"])
def test_loads_wait_for_their_scalar_operands(load, tmp_path):
    if not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("needs hipcc")
    src, asm = tmp_path / "probe.hip", tmp_path / "probe.s"
    src.write_text(SOURCE)
    subprocess.run([build.hipcc(), *build.COMMON, *build.DEVICE, f"-DLOAD=mezo::{load}", "--cuda-device-only", "-S",
                    str(src), "-o", str(asm)], check=True, capture_output=True)
    text = asm.read_text()
    body = text[text.index("s_waitcnt"):text.index("s_endpgm")]
    instructions = [x.split(";")[0].strip() for x in body.splitlines()]
    instructions = [x for x in instructions if x and not x.startswith(".") and not x.endswith(":")]
    assert any("global_load_lds" in x for x in instructions)
    assert missing_waits(instructions) == []
