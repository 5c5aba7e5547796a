"""The 64-row attention kernel writes its matrix instructions in assembly, for which the compiler adds no waits: an operand that a vector
instruction wrote has to be two wait states old, and a result that one reads has to be finished.  Looked up in the assembly of this library's own
source (no GPU)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2605_06472_amd import build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not shutil.which("hipcc"):
        pytest.skip("needs hipcc")
    asm = str(tmp_path_factory.mktemp("asm") / "attn.s")
    subprocess.run(["hipcc", *build.FLAGS, "-w", "-S", "--cuda-device-only", os.path.join(build.CSRC, "attn_bf16.hip"), "-o", asm],
                   check=True, stderr=subprocess.DEVNULL)
    out = {}
    for m in re.finditer(r"^(\S*attn_bf16_w64_kernelI\S*):[^\n]*\n(.*?)^\.Lfunc_end", open(asm).read(), re.M | re.S):
        lines = (l.split(";")[0].strip() for l in m[2].splitlines())
        out[m[1]] = [l for l in lines if l and not l.startswith(".")]
    return out


def _registers(operand):
    m = re.fullmatch(r"([va])(?:\[(\d+):(\d+)\]|(\d+))", operand.strip())
    if not m:
        return set()
    first, last = (m[4], m[4]) if m[4] else (m[2], m[3])
    return {(m[1], i) for i in range(int(first), int(last) + 1)}


def violations(ops):
    """Matrix instructions that read a register less than two wait states after a vector instruction wrote it, and other instructions that read a matrix
    instruction's result within its 16 passes."""
    written, result, now, bad = {}, {}, 0, []
    for op in ops:
        name, _, rest = op.partition(" ")
        args = re.split(r",\s*(?![^\[]*\])", rest) if rest else []
        if name == "s_nop":
            now += int(args[0]) + 1
            continue
        now += 1
        if name.startswith("v_mfma"):
            if any(now - written.get(r, -9) - 1 < 2 for a in args[1:] for r in _registers(a)):
                bad.append(op)
            for r in _registers(args[0]):
                written.pop(r, None)
                result[r] = now + 3                      # (its issue takes four)
            now += 3
            continue
        reads = args if name.startswith(("ds_write", "global_store", "buffer_store")) else args[1:]
        if any(now - result.get(r, -99) < 18 for a in reads for r in _registers(a)):
            bad.append(op)
        for r in _registers(args[0]) if args else ():
            result.pop(r, None)
            if name.startswith("v_"):
                written[r] = now
            else:
                written.pop(r, None)
    return bad


def test_operands_are_there_when_they_are_read(kernels):
    names = [n for n in kernels if n.endswith("Lb1EEEvNS_10AttnParamsEi")]
    assert len(names) == 4, sorted(kernels)
    for name in names:
        ops = kernels[name]
        assert sum(op.startswith("v_mfma") for op in ops) >= 64
        assert violations(ops) == [], name
        assert not any(op.startswith("scratch_") for op in ops), name


def test_a_late_operand_is_seen():
    ops = ["v_accvgpr_read_b32 v5, a3", "s_nop 0", "v_mfma_f32_32x32x16_bf16 v[16:31], v[0:3], v[4:7], v[16:31]"]
    assert violations(ops)
    assert not violations([ops[0], "s_nop 1", ops[2]])
    assert violations([ops[2], "v_max_f32_e32 v40, v17, v18"]) and not violations([ops[2], "s_nop 15", "s_nop 3", "v_max_f32_e32 v40, v17, v18"])
