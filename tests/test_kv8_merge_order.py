"""The 8-bit decode kernel that merges in its last work-group relies on the order of its instructions, as the bf16 one does: partials stored past the
XCD's L2, a wait until they are done, a barrier, and only then the count that lets another work-group read them.  Looked up in the
assembly of this library's own source (no GPU)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2605_06472_amd import build


def test_partials_are_written_through_before_the_count(tmp_path):
    if not shutil.which("hipcc"):
        pytest.skip("needs hipcc")
    asm = str(tmp_path / "decode.s")
    subprocess.run(["hipcc", *build.FLAGS, "-w", "-S", "--cuda-device-only", os.path.join(build.CSRC, "decode_kv8.hip"), "-o", asm],
                   check=True, stderr=subprocess.DEVNULL)
    kernels = {m[1]: m[2] for m in re.finditer(r"^(\S*decode_kv8_kernelI\S*):(.*?)^\.Lfunc_end", open(asm).read(), re.M | re.S)}
    assert len(kernels) == 8
    for name, body in kernels.items():
        ops = [l for l in (l.split(";")[0].strip() for l in body.splitlines()) if l and not l.startswith(".")]
        counts = [i for i, l in enumerate(ops) if l.startswith("global_atomic_inc")]
        fused = re.search(r"ILi\d+ELb1E", name) is not None
        assert len(counts) == fused, name
        if not fused:
            continue
        near = [l for l in ops[:counts[0]] if re.match(r"global_store|s_barrier|s_waitcnt vmcnt\(0\)", l)]
        last = max(i for i, l in enumerate(near) if l.startswith("global_store") and l.endswith("sc1"))
        assert near[last + 1:][:2] == ["s_waitcnt vmcnt(0)", "s_barrier"], (name, near[-8:])
        assert not any(l.startswith("global_store") for l in near[last + 1:]), name
        # and the reader drops what its own caches hold before the first load of a partial
        reader = [l for l in ops[counts[0]:] if re.match(r"buffer_inv sc1|global_load", l)]
        assert reader[0].startswith("buffer_inv sc1"), name
