"""Registers of attention over the cache (compiled for the device here, no GPU needed): private memory in its loops waits for the loads on their way."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1810_08723_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_private_memory():
    """None but a few values that are kept outside the loops over whole tiles: of 256 channels and few rows, and of 128 channels and many rows of floats.  An array
    with an index that is not known when this is compiled would lie there (of 64 channels and many rows: 48 bytes a lane, written and read for every tile)."""
    from paper_1810_08723_amd.build import COMMON
    r = subprocess.run([HIPCC, *COMMON, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-x", "hip", "-c",
                        os.path.join(CSRC, "cache_attention.hip"), "-o", os.devnull], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    private = [int(n) for n in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)]
    waves = [int(n) for n in re.findall(r"Occupancy \[waves/SIMD\]: (\d+)", r.stderr)]
    assert len(names) == len(private) == len(waves) == 30
    for name, size, occupancy in zip(names, private, waves):
        few = "16attention_kernel" in name
        spills = (few and "ILi256ELi1EDF16" in name) or "attention_many_kernelILi128ELi2Ef" in name
        assert size <= (24 if spills else 0), (name, size)
        if "attention_many_kernel" in name or (few and "DF16" in name):
            assert occupancy >= (3 if few and ("ILi64ELi1E" in name or "ILi128ELi1E" in name) else 2), (name, occupancy)
