"""Direct loads from memory to LDS (global_load_lds) are issued from inline asm, where the
compiler inserts no wait states.  The hardware wants five between a vector instruction that
writes a scalar register (v_readfirstlane, say) and a vector-memory instruction that reads
it, and one between a write of M0 and a load to LDS.  Counted here in the machine code of
every kernel that was built."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_39056_amd import _build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
BASE_STATES, M0_STATES = 5, 1


def registers(text):
    """Scalar registers that an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", text)
    if m:
        return {f"s{i}" for i in range(int(m.group(1)), int(m.group(2)) + 1)}
    if text == "vcc":
        return {"vcc_lo", "vcc_hi"}
    return {text} if re.fullmatch(r"s\d+|vcc_lo|vcc_hi|m0", text) else set()


def written(name, operands):
    """Scalar registers that a vector or scalar instruction writes, or may write."""
    if name.startswith("s_"):
        return registers(operands[0]) if operands else set()
    out = registers(operands[0]) if operands else set()
    if len(operands) > 1 and re.match(r"v_(add|sub|subrev|addc|subb|subbrev)_co|v_mad_[ui]64|v_div_scale", name):
        out |= registers(operands[1])
    return out


def faults(lines):
    """Direct loads in a listing, and what is wrong with some of them."""
    loads, wrong = 0, []
    code = []  # (name, operands); None where another path may come in
    for line in lines:
        if re.match(r"[0-9a-f]+ <", line):
            code = [None]
        m = re.match(r"\s+([a-z]\w+)\s*([^/]*?)\s*(//|$)", line)
        if not m:
            continue
        name, operands = m.group(1), [o.strip().split(" ")[0] for o in m.group(2).split(",")] if m.group(2) else []
        code.append((name, operands))
        if not re.match(r"(global|buffer)_load_lds", name) and " lds" not in m.group(2):
            continue
        loads += 1
        need = set().union(*(registers(o) for o in operands)) - {"m0"}
        states, at = 0, len(code) - 2
        while states < max(BASE_STATES, M0_STATES):
            if code[at] is None or code[at][0].startswith(("s_cbranch", "s_branch")):
                wrong.append((states, "branch", line.strip()))
                break
            before, ops = code[at]
            out = written(before, ops)
            if before.startswith("v_") and out & need and states < BASE_STATES:
                wrong.append((states, f"{before} {ops[0]}", line.strip()))
                break
            if "m0" in out and states < M0_STATES:
                wrong.append((states, f"{before} m0", line.strip()))
                break
            states += int(ops[0], 0) + 1 if before == "s_nop" else 1
            at -= 1
    return loads, wrong


def test_the_count_itself():
    def listing(*code):
        return ["0000 <kernel>:"] + ["\ts_mov_b32 s9, 0 // 0: 0"] * 6 + [f"\t{c} // 0: 0" for c in code]

    load = "global_load_lds_dwordx4 v1, s[0:1]"
    assert faults(listing("v_readfirstlane_b32 s1, v3", "s_mov_b32 m0, s2", "s_nop 3", load)) == (1, [])
    assert faults(listing("v_readfirstlane_b32 s2, v3", "s_mov_b32 m0, s2", "s_nop 0", load)) == (1, [])
    assert faults(listing("v_mov_b32_e32 v1, v3", "s_mov_b32 m0, s2", "s_nop 0", "global_load_lds_dwordx4 v[1:2], off")) == (1, [])
    for bad in (["v_readfirstlane_b32 s1, v3", "s_mov_b32 m0, s2", "s_nop 2", load],
                ["v_readfirstlane_b32 s0, v3", "v_mov_b32_e32 v4, v3", "s_mov_b32 m0, s2", "s_nop 0", load],
                ["v_mad_u64_u32 v[4:5], s[0:1], v2, v3, 0", "s_mov_b32 m0, s2", "s_nop 0", load],
                ["s_mov_b32 m0, s2", load], ["s_mov_b32 m0, s2", "s_nop 0", "s_cbranch_scc0 4", load]):
        assert len(faults(listing(*bad))[1]) == 1


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    if not os.path.exists(_build.LIB):
        _build.build()
    d = tmp_path_factory.mktemp("code")
    shutil.copy(_build.LIB, d / "sq.so")
    subprocess.run([OBJDUMP, "--offloading", "sq.so"], cwd=d, check=True, capture_output=True)
    return [str(p) for p in sorted(d.iterdir()) if p.name.endswith(_build.ARCH) and p.stat().st_size > 0]


def test_direct_loads_have_their_wait_states(kernels):
    loads, wrong = 0, []
    for path in kernels:
        text = subprocess.run([OBJDUMP, "-d", path], check=True, capture_output=True, text=True).stdout
        n, w = faults(text.splitlines())
        loads, wrong = loads + n, wrong + w
    assert loads > 1000
    assert not wrong, f"{len(wrong)} of {loads}: {wrong[:3]}"
