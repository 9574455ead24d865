"""What the operators' kernels hold in registers, from the assembly text (no GPU needed): none uses scratch memory but those of the norms that are
named in radial_norm.hip, rows of more than 8192 channels and, by eight bytes, gradients of float32 rows of more than 4096."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_19852_amd import build as hip_build


@pytest.fixture(scope="module")
def scratch(tmp_path_factory):
    """{source: {kernel: bytes of scratch memory for each lane}}"""
    if not os.path.exists(hip_build.HIPCC) and shutil.which(hip_build.HIPCC) is None:
        pytest.skip("hipcc not available")
    to = tmp_path_factory.mktemp("asm")
    running = {}
    for name in ("radial_norm", "radial_rope", "radial_product"):
        cmd = [hip_build.HIPCC, *hip_build.FLAGS, "--cuda-device-only", "-S", os.path.join(hip_build.CSRC, name + ".hip"), "-o", str(to / (name + ".s"))]
        running[name] = subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = {}
    for name, p in running.items():
        text, _ = p.communicate()
        assert p.returncode == 0, text[-3000:]
        sizes = re.findall(r"\.amdhsa_kernel (\S+).*?\.amdhsa_private_segment_fixed_size (\d+)", (to / (name + ".s")).read_text(), re.S)
        out[name] = {kernel: int(size) for kernel, size in sizes}
    return out


@pytest.mark.parametrize("source, kernels", [("radial_rope", 7), ("radial_product", 42)])
def test_rope_and_product_use_no_scratch_memory(scratch, source, kernels):
    assert len(scratch[source]) == kernels and not any(scratch[source].values()), scratch[source]


def test_norms_use_scratch_memory_only_where_they_say(scratch):
    found = scratch["radial_norm"]
    rows = {k: re.search(r"norm_(fwd|bwd)_kernelI(f|DF16b)(f|DF16b|S\w*_)Lb([01])ELi(\d)ELb([01])", k) for k in found}
    assert sum(m is not None for m in rows.values()) == 2 * 4 * 2 * 6 and len(found) == 2 * 4 * 2 * 6 + 3
    for kernel, m in rows.items():
        if m and m[5] == "4":
            assert found[kernel] <= (100 if m[1] == "fwd" else 800), (kernel, found[kernel])
        elif m and (m[1], m[2], m[3], m[4], m[5]) == ("bwd", "f", "f", "1", "2"):
            assert found[kernel] <= 8, kernel
        else:
            assert found[kernel] == 0, (kernel, found[kernel])
