"""Host-side checks of what the compiler made of the operators' kernels: the wait states around inline assembly, and that no kernel
spills more than a handful of vector registers. (The MFMAs of ficco_direct.hip are the compiler's own, which counts the states
behind them by the instruction's passes; the check is for the longest.)"""
import os
import re
import subprocess

import pytest

from paper_2512_10236_amd import _build
from test_asm_hazards import hazards

# today: 0-4
MAX_VGPR_SPILL = 16


@pytest.mark.parametrize("src,mfmas", [("ficco_linear.hip", 500), ("ficco_linear_strided.hip", 1000), ("ficco_direct.hip", None), ("ficco_norm.hip", 0), ("ficco_balance.hip", 0)])
def test_wait_states_and_spills(src, mfmas, tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    out = str(tmp_path / "k.s")
    cmd = [hipcc] + _build.FLAGS + ["-S", "--cuda-device-only", os.path.join(_build.CSRC, src), "-o", out, "-Rpass-analysis=kernel-resource-usage"]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-2000:]
    name, spills = None, {}
    for line in r.stdout.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            name = m.group(1)
        m = re.search(r"VGPRs Spill: (\d+)", line)
        if m:
            spills[name] = int(m.group(1))
    assert spills, "the compiler printed no resource usage"
    assert not {k: v for k, v in spills.items() if v > MAX_VGPR_SPILL}
    if mfmas is None:
        return
    with open(out) as f:
        bad, seen = hazards(f.read())
    assert seen >= mfmas, "MFMAs in the assembly"
    assert not bad, "\n".join(map(str, sorted(bad)[:20]))
