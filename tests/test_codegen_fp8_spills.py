"""Registers of the kernels in 8-bit floating point and of sampling (no GPU needed): none spills but those known to, and these no
more than they do."""
import os
import re
import subprocess

import pytest

SOURCES = ("attention8.hip", "kv8.hip", "product_fp8.hip", "sample.hip")
# Bytes of scratch a lane, vector registers and scalar registers that are spilled (the latter go to lanes of vector registers), at
# most.  Heads of 128 and many columns keep 168 registers for three waves a SIMD; sampling's 1024 threads leave 128 each.
KNOWN = [(r"attention8_wide_kernelIDF16_Li128", 48, 11, 0), (r"attention8_wide_kernelIDF16bLi128", 12, 2, 0),
         (r"sample_kernelIf", 128, 30, 134), (r"sample_kernelIDF16b?_?E", 64, 11, 130), (r"kv8_append_kernelIDF16(_|b)Li128", 0, 0, 74)]


@pytest.fixture(scope="module")
def kernels():
    from paper_2606_15652_amd import build
    out = {}
    for src in build.sources():
        if os.path.basename(src) not in SOURCES:
            continue
        cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *[f for f in build.compile_flags(src) if f != "-fPIC"],
               "--cuda-device-only", "-S", src, "-o", "-"]
        text = subprocess.run(cmd, capture_output=True, text=True, check=True).stdout
        text = text[text.index(".amdgpu_metadata"):]
        for part in re.split(r"(?m)^  - \.", text)[1:]:
            name = re.search(r"\.name: +(_Z\S+)", part).group(1)
            out[name] = [int(re.search(rf"\.{key}: +(\d+)", part).group(1))
                         for key in ("private_segment_fixed_size", "vgpr_spill_count", "sgpr_spill_count")]
    return out


def test_spills(kernels):
    assert len(kernels) >= 2 * 11 + 1 + 8 + 3 * 13 + 3
    met = set()
    for name, used in kernels.items():
        most = [0, 0, 0]
        for i, (pattern, *known) in enumerate(KNOWN):
            if re.search(pattern, name):
                most = known
                met.add(i)
        assert all(u <= m for u, m in zip(used, most)), (name, used, most)
    assert len(met) == len(KNOWN)
