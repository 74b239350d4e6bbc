"""Registers of attention over whole sequences (compiled for the device here, no GPU needed): two wavefronts to a SIMD, and no private memory in loops over tiles of whole rows."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1810_08723_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FORWARD = ["attention_rows_kernel<{t}, 64, true, 4, 64>({a})", "attention_rows_kernel<{t}, 80, true, 8, 64>({a})", "attention_rows_kernel<{t}, 128, true, 8, 64>({a})",
           "attention_rows_kernel<{t}, 192, true, 4, 32>({a})", "attention_few_kernel<{t}, 64, true>({a})", "attention_few_kernel<{t}, 128, true>({a})"]
BACKWARD = ["attention_queries_kernel<{t}, 64, true, 4, 64>({a}, f32x2 *, f32x2 *)", "attention_queries_kernel<{t}, 128, true, 4, 64>({a}, f32x2 *, f32x2 *)",
            "attention_keys_kernel<{t}, 64, true, 4>({a}, const f32x2 *, const f32x2 *)", "attention_keys_kernel<{t}, 128, true, 8>({a}, const f32x2 *, const f32x2 *)"]


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
@pytest.mark.parametrize("header,kernels", [("attention_forward.hpp", FORWARD), ("attention_backward.hpp", BACKWARD)], ids=["forward", "gradient"])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_private_memory_and_wavefronts(header, kernels, kind, tmp_path):
    from paper_1810_08723_amd.build import COMMON
    made = " ".join(f"template __global__ void {k.format(t=kind, a='const AttentionArgs, uint32_t')};" for k in kernels)
    source = tmp_path / "kernels.hip"
    source.write_text(f'#include "{os.path.join(CSRC, header)}"\nnamespace ocn {{ namespace {{ {made} }} }}\n')
    r = subprocess.run([HIPCC, *COMMON, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-x", "hip", "-c", str(source), "-o", os.devnull],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    private = [int(n) for n in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)]
    waves = [int(n) for n in re.findall(r"Occupancy \[waves/SIMD\]: (\d+)", r.stderr)]
    found = [x for x in zip(names, private, waves) if "order" not in x[0]]
    assert len(found) == len(kernels)
    for name, size, occupancy in found:
        assert size == 0 and occupancy >= 2, (name, size, occupancy)
