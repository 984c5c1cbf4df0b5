"""Registers of the kernels for positions and contexts in 4 bits, as the compiler reports them (no GPU): none spills or keeps an
array in scratch memory (a register array indexed by a lane's number once cost every attention launch 14 us), and as many
wavefronts of an attention kernel fit a SIMD as its launch bounds were chosen for."""
import os
import re
import subprocess

import pytest

from paper_2502_01960_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
WAVES = {("DF16b", "128", "1", "1"): 4, ("DF16b", "128", "0", "1"): 3, ("DF16b", "128", "0", "2"): 2,     # type, D, narrow, tiles
         ("f", "128", "0", "1"): 3, ("f", "64", "0", "1"): 4}


def _report(source, tmp_path):
    cmd = [HIPCC, *build.FLAGS, "--offload-device-only", "-Rpass-analysis=kernel-resource-usage", "-x", "hip", "-c",
           os.path.join(build.CSRC, source), "-o", str(tmp_path / "kernels.o")]
    text = subprocess.run(cmd, check=True, capture_output=True, text=True, timeout=600).stderr
    field = lambda body, name: int(re.search(name + r"[^:]*: (\d+)", body).group(1))
    return {name: {f: field(body, f) for f in ("ScratchSize", "Occupancy", "SGPRs Spill", "VGPRs Spill")}
            for name, body in re.findall(r"Function Name: (\S+)(.*?)(?=Function Name:|\Z)", text, re.S)}


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
@pytest.mark.parametrize("source,n", [("q4_attn.hip", 14), ("q4.hip", 6), ("position.hip", 12)])
def test_nothing_is_spilled(source, n, tmp_path):
    report = _report(source, tmp_path)
    assert len(report) == n, sorted(report)
    for name, r in report.items():
        assert (r["ScratchSize"], r["SGPRs Spill"], r["VGPRs Spill"]) == (0, 0, 0), name
    waves = {m.groups(): r["Occupancy"] for name, r in report.items()
             for m in [re.search(r"5ShapeI(DF16b|f)Li(\d+)ELb(\d)ELi(\d)E", name)] if m}
    assert waves == (WAVES if source == "q4_attn.hip" else {})
