"""No kernel of the sources with flags of their own keeps registers in scratch memory, compiled as the library is."""

from __future__ import annotations

import os
import re
import subprocess

import pytest

from paper_2607_21848_amd import build as B


@pytest.mark.parametrize("source", B.WIDE_SOURCES)
def test_no_scratch(source, tmp_path):
    try:
        cc = B.hipcc()
    except RuntimeError as e:
        pytest.skip(str(e))
    out = subprocess.run([cc, *B.compile_flags(), *B.WIDE_FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-x", "hip",
                          "-c", os.path.join(B.CSRC, source), "-o", str(tmp_path / "device.o")], check=True, capture_output=True, text=True).stderr
    kernels = re.findall(r"Function Name: (\S+)", out)
    assert kernels and len(kernels) == len(set(kernels))
    for what in (r"ScratchSize \[bytes/lane\]", "SGPRs Spill", "VGPRs Spill"):
        figures = [int(x) for x in re.findall(what + r": (\d+)", out)]
        assert len(figures) == len(kernels) and not any(figures), list(zip(kernels, figures))


def test_every_source_is_built():
    """No kernel source lies beside the lists that the build reads."""
    there = {f for f in os.listdir(B.CSRC) if f.endswith((".hip", ".cpp"))}
    assert there == set(B.SOURCES) | set(B.WIDE_SOURCES) and len(there) == len(B.SOURCES) + len(B.WIDE_SOURCES)
