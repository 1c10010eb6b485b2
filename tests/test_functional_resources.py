"""Register budget of the rotary, attention and distillation kernels (CPU only: a compile, no
launch).

The attention kernels keep score tiles, the rows' fragments and their sums in registers
beside copies in flight to LDS; the distillation keeps whole rows.  A spilled register or a
private array becomes scratch traffic that shares the vector-memory counter with those copies,
so every kernel must use no scratch memory and spill no VGPR, and the attention kernels must
leave room for two waves on a SIMD."""
import functools
import os
import re
import subprocess
import sys
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@functools.lru_cache(maxsize=None)
def _kernels(unit):
    sys.path.insert(0, ROOT)
    from paper_2410_15352_amd import build as B
    try:
        hipcc = B.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    with tempfile.TemporaryDirectory(prefix="compact_res_") as d:
        cmd = [hipcc, *B.FLAGS, *dict(B.UNITS)[unit], "-I", B.INCLUDE, "--offload-device-only", "-S",
               os.path.join(B.CSRC, unit), "-o", os.path.join(d, "u.s"), "-Rpass-analysis=kernel-resource-usage"]
        res = subprocess.run(cmd, capture_output=True, text=True, cwd=d)
        assert res.returncode == 0, res.stderr[-2000:]
    kernels, cur = {}, None
    for line in res.stderr.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            cur = kernels.setdefault(m.group(1), {})
            continue
        m = re.search(r"remark:\s+([A-Za-z ]+?)(?: \[[^\]]*\])?: (\d+) \[", line)
        if m and cur is not None:
            cur[m.group(1).strip()] = int(m.group(2))
    return kernels


# unit -> kernels it must hold
KERNELS = {
    "rotary.hip": ("k_rotary",),
    "attention.hip": ("k_attn_fwd", "k_attn_split", "k_attn_join", "k_attn_dq", "k_attn_dkvI", "k_attn_dkv_sum"),
    "distill.hip": ("k_distill",),
}


@pytest.mark.parametrize("unit", list(KERNELS))
def test_kernels_use_no_scratch(unit):
    kernels = _kernels(unit)
    for name in KERNELS[unit]:
        assert any(name in k for k in kernels), f"no {name} in {unit}"
    for name, use in kernels.items():
        assert use["ScratchSize"] == 0 and use["VGPRs Spill"] == 0, (name, use)


def test_two_waves_of_attention_on_a_simd():
    for name, use in _kernels("attention.hip").items():
        assert use["Occupancy"] >= 2, (name, use)
