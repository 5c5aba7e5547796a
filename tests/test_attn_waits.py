"""The 64-row attention kernel over an 8-bit pool writes its matrix instructions in assembly, for which the compiler adds no waits: an operand that a
vector instruction wrote has to be two wait states old when a matrix instruction reads it, and a matrix instruction's result
finished (11 for eight passes; 18 asked for) when anything but the next sum of the same chain does; the exponentials' results may not be read by the very next
instruction.  Looked up in the assembly of this library's own source, along every path through it (no GPU)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2605_06472_amd import build

WAITS, RESULT, FORGET = 2, 18, 40


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not shutil.which("hipcc"):
        pytest.skip("needs hipcc")
    asm = str(tmp_path_factory.mktemp("asm") / "attn.s")
    subprocess.run(["hipcc", *build.FLAGS, "-w", "-S", "--cuda-device-only", os.path.join(build.CSRC, "attn_bf16.hip"), "-o", asm],
                   check=True, stderr=subprocess.DEVNULL)
    return {m[1]: m[2].splitlines() for m in re.finditer(r"^(\S*attn_bf16_w64_kernelI\S*):[^\n]*\n(.*?)^\.Lfunc_end", open(asm).read(), re.M | re.S)}


def _registers(operand):
    m = re.fullmatch(r"([va])(?:\[(\d+):(\d+)\]|(\d+))", operand.strip())
    if not m:
        return set()
    first, last = (m[4], m[4]) if m[4] else (m[2], m[3])
    return {(m[1], i) for i in range(int(first), int(last) + 1)}


def _blocks(lines):
    """[(label, instructions)], and the blocks that each may go on to."""
    blocks = [("", [])]
    for l in lines:
        l = l.split(";")[0].strip()
        label = re.match(r"(\.LBB\S+):", l)
        if label:
            blocks.append((label[1], []))
        elif l and not l.startswith("."):
            blocks[-1][1].append(l)
            if l.startswith(("s_cbranch", "s_branch", "s_endpgm")):
                blocks.append(("", []))
    at = {b[0]: i for i, b in enumerate(blocks)}
    after = []
    for i, (_, ops) in enumerate(blocks):
        last = ops[-1] if ops else ""
        to = [at[last.split()[1]]] if last.startswith(("s_cbranch", "s_branch")) else []
        if not last.startswith(("s_branch", "s_endpgm")) and i + 1 < len(blocks):
            to.append(i + 1)
        after.append(to)
    return blocks, after


def _run(ops, written, result, bad=None):
    """Ages (in wait states, negative: before the block) of vector results and of matrix results behind the block."""
    written, result, now, trans = dict(written), dict(result), 0, set()
    for op in ops:
        name, _, rest = op.partition(" ")
        args = re.split(r",\s*(?![^\[]*\])", rest) if rest else []
        if name == "s_nop":
            now, trans = now + int(args[0]) + 1, set()
            continue
        now += 1
        if name.startswith("v_mfma"):
            if bad is not None:
                late = any(now - written.get(r, -99) - 1 < WAITS for a in args[1:4] for r in _registers(a))
                unfinished = any(now - result.get(r, -99) < RESULT for a in args[1:3] + [a for a in args[3:4] if a != args[0]] for r in _registers(a))
                if late or unfinished:
                    bad.append(op)
            for r in _registers(args[0]):
                written.pop(r, None)
                result[r] = now + 3                      # (its issue takes four)
            now, trans = now + 3, set()
            continue
        reads = args if name.startswith(("ds_write", "global_store", "buffer_store")) else args[1:]
        read = set().union(*(_registers(a) for a in reads)) if reads else set()
        if bad is not None and (any(now - result.get(r, -99) < RESULT for r in read) or (read & trans and not name.startswith(("v_exp", "v_rcp")))):
            bad.append(op)
        trans = _registers(args[0]) if name.startswith(("v_exp", "v_rcp")) else set()
        if args and not name.startswith(("ds_write", "global_store", "buffer_store", "s_")):
            for r in set().union(_registers(args[0]), _registers(args[1]) if name.startswith("v_permlane") else set()):
                if bad is not None and now - result.get(r, -99) < RESULT:
                    bad.append(op)
                result.pop(r, None)
                if name.startswith("v_"):
                    written[r] = now
                else:
                    written.pop(r, None)
    return [{k: v - now for k, v in d.items() if now - v < FORGET} for d in (written, result)]


def violations(lines):
    blocks, after = _blocks(lines)
    state, todo = {0: [{}, {}]}, [0]
    while todo:
        i = todo.pop()
        out = _run(blocks[i][1], *state[i])
        for n in after[i]:
            if n not in state:
                state[n] = [dict(d) for d in out]
                todo.append(n)
                continue
            newer = [(d, k, v) for d, e in zip(state[n], out) for k, v in e.items() if v > d.get(k, -99)]
            for d, k, v in newer:
                d[k] = v
            if newer:
                todo.append(n)
    bad = []
    for i, s in state.items():
        _run(blocks[i][1], *s, bad)
    return bad


def test_operands_are_there_when_they_are_read(kernels):
    names = [n for n in kernels if n.endswith("Lb1EEEvNS_10AttnParamsEi")]
    assert len(names) == 4, sorted(kernels)
    for name in names:
        assert sum("v_mfma" in l for l in kernels[name]) >= 64
        assert violations(kernels[name]) == [], name
        assert not any(l.strip().startswith("scratch_") for l in kernels[name]), name


def test_what_comes_too_early_is_seen():
    read, mfma = "v_accvgpr_read_b32 v5, a3", "v_mfma_f32_32x32x16_bf16 v[16:31], v[0:3], v[4:7], v[16:31]"
    assert violations([read, "s_nop 0", mfma]) and not violations([read, "s_nop 1", mfma])
    assert violations([mfma, "v_max_f32_e32 v40, v17, v18"]) and not violations([mfma, "s_nop 15", "s_nop 3", "v_max_f32_e32 v40, v17, v18"])
    assert violations([mfma, "s_branch .LBB0_2", ".LBB0_1:", "s_endpgm", ".LBB0_2:", "v_mov_b32_e32 v40, v17"])
    assert violations([".LBB0_1:", "v_mov_b32_e32 v40, v17", mfma, "s_cbranch_scc0 .LBB0_1"])
    assert violations(["v_exp_f32 v1, v2", "v_add_f32_e32 v3, v1, v1"]) and not violations(["v_exp_f32 v1, v2", "s_nop 0", "v_add_f32_e32 v3, v1, v1"])
