"""What the kernels of the integer products and of AdamW hold in registers, from the assembly text (no GPU needed): none uses scratch memory, and the product's
loops hold all sums where the matrix instructions want them."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_19852_amd import build as hip_build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{source: {kernel: (bytes of scratch memory for each lane, text)}}"""
    if not os.path.exists(hip_build.HIPCC) and shutil.which(hip_build.HIPCC) is None:
        pytest.skip("hipcc not available")
    to = tmp_path_factory.mktemp("asm")
    running = {}
    for name in ("radial_quantize_i8", "radial_product_i8", "radial_adamw"):
        cmd = [hip_build.HIPCC, *hip_build.FLAGS, "--cuda-device-only", "-S", os.path.join(hip_build.CSRC, name + ".hip"), "-o", str(to / (name + ".s"))]
        running[name] = subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = {}
    for name, p in running.items():
        said, _ = p.communicate()
        assert p.returncode == 0, said[-3000:]
        text = (to / (name + ".s")).read_text()
        sizes = dict(re.findall(r"\.amdhsa_kernel (\S+).*?\.amdhsa_private_segment_fixed_size (\d+)", text, re.S))
        out[name] = {k: (int(v), text[text.index(f"\n{k}:"):text.index(".Lfunc_end", text.index(f"\n{k}:"))]) for k, v in sizes.items()}
    return out


@pytest.mark.parametrize("source, count", [("radial_quantize_i8", 2 * (6 + 3 + 2) + 1), ("radial_product_i8", 10 + 1 + 6), ("radial_adamw", 5)])
def test_no_scratch_memory(kernels, source, count):
    assert len(kernels[source]) == count and not any(size for size, _ in kernels[source].values()), {k: v[0] for k, v in kernels[source].items()}


def test_sums_of_a_product_are_not_moved(kernels):
    """Without a bound on the waves of a SIMD, workgroups of four waves get some of their sums in registers that only matrix instructions reach, and moved them in and out: 84 moves
    beside 32 matrix instructions a stage."""
    tiles = {k: text for k, (_, text) in kernels["radial_product_i8"].items() if "tile_kernel" in k}
    assert len(tiles) == 10 and not any("accvgpr" in text for text in tiles.values())


def test_a_step_uses_no_library_division(kernels):
    """The sequences of a correctly rounded division scale their operands; the step's quotients do without."""
    step = [text for k, (_, text) in kernels["radial_adamw"].items() if "adamw_step" in k]
    # what is left: the bias corrections of a step counted on the device
    assert len(step) == 2 and all(text.count("v_div_fixup_f32") <= 2 for text in step), [text.count("v_div_fixup_f32") for text in step]
