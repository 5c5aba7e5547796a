"""The 64-row attention kernel over bf16 pools, whose matrix instructions are assembly statements too: the same waits as over 8-bit pools (no GPU)."""
from tests.test_attn_waits import kernels, violations             # noqa: F401


def test_operands_are_there_when_they_are_read(kernels):           # noqa: F811
    names = [n for n in kernels if n.endswith("Lb0EEEvNS_10AttnParamsEi")]
    assert len(names) == 4, sorted(kernels)
    for name in names:
        assert sum("v_mfma" in l for l in kernels[name]) >= 64
        assert violations(kernels[name]) == [], name
        assert not any(l.strip().startswith("scratch_") for l in kernels[name]), name
